"""GPU tests of focus_token_logprobs / focus_token_logprobs_bwd against the definition in float64.

Bounds. Exponents d = (z - m) log2 e are fp32, their error 2^-24 |d| log2-units, so a term is good to 2^-24 (|d| + 2) and
sums of positive terms, in chains of at most V / 512 / 8 steps, to about 1e-5 relative: lse is held to 1e-5 + 2^-22 |lse|,
logp and the alternatives to the same with |z| in it, the entropy (a quotient of two such sums) to 4e-5 (1 + entropy). The
gradient's probabilities carry the rounding of lse in their exponent: 4e-6 (1 + |lse| + |log p|) relative, times the larger of
its two terms; bf16 results add half a unit in the last place.
"""
import math

import pytest
import torch

from gpu_common import announce, require_gpu

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def F():
    return require_gpu()


def reference(Z, target, top):
    z = Z.double().cpu()
    # relative to the row's largest logit, whose size can exceed the digits that a sum with log V has
    m = z.amax(1, keepdim=True)
    none = torch.isneginf(m)[:, 0]
    z = z - torch.where(none[:, None], 0.0, m)
    rest = torch.logsumexp(z, 1)
    lse = torch.where(none, -math.inf, m[:, 0] + rest)
    lp = torch.where(none[:, None], -math.inf, z - torch.where(none, 0.0, rest)[:, None])
    p = lp.exp()
    ent = -torch.where(p > 0, p * lp.clamp(min=-1e300), 0.0).sum(1)
    t = target.cpu()
    logp = torch.where(t < 0, 0.0, lp.gather(1, t.clamp(min=0)[:, None])[:, 0])
    order = torch.sort(Z.float().cpu() + 0.0, dim=1, descending=True, stable=True)[1][:, :top]
    return lse, logp, ent, lp, order


def check(F, Z, target, top):
    T, V = Z.shape
    ws = F.workspace(F.token_logprobs_workspace_size(T, V, top))
    logp, ent, lse, top_logp, top_index = F.token_logprobs(Z, target, top, ws=ws)
    assert F.check_flags(ws) == F.OK
    rl, rp, re, lp, order = reference(Z, target, top)
    none = torch.isneginf(rl)
    same = lambda got, ref, lim: bool((((got - ref).abs() <= lim) | (got == ref)).all())
    assert same(lse.double().cpu(), rl, 1e-5 + 2.0 ** -22 * rl.abs())
    assert same(ent.double().cpu(), re, 4e-5 * (1 + re))
    zt = Z.double().cpu().gather(1, target.cpu().clamp(min=0)[:, None])[:, 0]
    assert same(logp.double().cpu(), rp, 1e-5 + 2.0 ** -22 * (rl.abs() + zt.abs()))
    n = min(top, V)
    if top:
        assert torch.equal(top_index[:, :n].cpu().long(), order[:, :n])
        assert (top_index[:, n:] == -1).all() and torch.isneginf(top_logp[:, n:]).all()
        rt = lp.gather(1, order)
        assert same(top_logp[:, :n].double().cpu(), rt, 1e-5 + 2.0 ** -22 * (rl.abs()[:, None] + rt.abs()))
    return lse, ent, lp, none


def logits(T, V, dt, seed, scale=2.5):
    return (torch.randn(T, V, generator=torch.Generator().manual_seed(seed)) * scale).to(DT[dt]).cuda()


def targets(T, V, seed):
    g = torch.Generator().manual_seed(seed)
    t = torch.randint(0, V, (T,), generator=g)
    t[torch.rand(T, generator=g) < 0.2] = -1
    return t.cuda()


SHAPES = [(1, 1), (1, 2), (3, 7), (2, 63), (5, 1000), (1, 151936), (2, 151935), (7, 32003), (520, 4099), (600, 1025), (513, 20000)]


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("T,V", SHAPES)
def test_forward_and_backward(F, T, V, dt):
    announce(f"token_logprobs {dt} T={T} V={V}")
    Z, t = logits(T, V, dt, V + T), targets(T, V, T)
    for top in (0, 1, 20):
        lse, ent, lp, _ = check(F, Z, t, top)
    g = torch.randn(T, generator=torch.Generator().manual_seed(1)).cuda()
    h = torch.randn(T, generator=torch.Generator().manual_seed(2)).cuda()
    for gl, he in ((g, None), (None, h), (g, h)):
        dZ = F.token_logprobs_bwd(Z, t, lse, ent, gl, he)
        p = lp.exp()
        gd = torch.zeros(T, 1, dtype=torch.float64) if gl is None else torch.where(t < 0, 0.0, gl).double().cpu()[:, None]
        hd = torch.zeros(T, 1, dtype=torch.float64) if he is None else he.double().cpu()[:, None]
        H = -(p * lp).sum(1, keepdim=True)
        ref = -p * (gd + hd * (lp + H))
        ref.scatter_add_(1, t.cpu().clamp(min=0)[:, None], gd)
        size = p * (gd.abs() + hd.abs() * (lp.abs() + H + 1))
        lim = 4e-6 * (1 + lse.double().cpu().abs()[:, None] + lp.abs()) * size + 2.0 ** -23 * ref.abs() + 1e-36
        if dt == "bf16":
            lim += 2.0 ** -8 * ref.abs()
        d = (dZ.double().cpu() - ref).abs()
        # the target's element is a difference of g and its part
        lim.scatter_add_(1, t.cpu().clamp(min=0)[:, None], 2.0 ** -22 * gd.abs())
        assert (d <= lim).all(), float((d / lim).max())


@pytest.mark.parametrize("top", [1, 2, 5, 33, 64])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_alternatives_of_many_kinds(F, dt, top):
    """Equal logits, rising and falling rows, runs of large values that fall to few threads, few distinct values."""
    g = torch.Generator().manual_seed(3)
    for V in (top + 3, 4096, 20011, 40000):
        i = torch.arange(V)
        rows = [torch.zeros(V), -i.float() / 64, i.float() / 64, torch.where(i % 4096 < 8, 5.0 + torch.randn(V, generator=g), -3.0),
                torch.where((i // 8) % 512 == 37, 9.0, 0.0), torch.randint(0, 3, (V,), generator=g).float(),
                torch.where((i // 8) % 512 < 3, torch.randn(V, generator=g).abs(), -1.0),
                torch.randn(V, generator=g) * torch.where(i % 2 == 0, 0.0, 1.0) * -1.0]
        Z = torch.stack(rows).to(DT[dt]).cuda()
        announce(f"alternatives {dt} V={V} top={top}")
        check(F, Z, targets(len(rows), V, 4), top)
        big = Z.repeat(70, 1)  # enough rows that each is one workgroup's
        check(F, big, targets(big.shape[0], V, 5), top)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_masked_logits(F, dt):
    """-inf logits: a masked vocabulary, rows with one token left, rows with none."""
    for T, V in ((6, 5000), (516, 3000), (2, 50)):
        Z = logits(T, V, dt, 9)
        Z[:, 100::3] = -math.inf
        Z[0] = -math.inf
        Z[1] = -math.inf
        Z[1, V // 2] = 3.0
        t = targets(T, V, 6)
        t[0] = 5
        lse, ent, lp, none = check(F, Z, t, 7)
        assert torch.isneginf(lse[0]) and ent[0] == 0 and ent[1] == 0
        g = torch.ones(T).cuda()
        dZ = F.token_logprobs_bwd(Z, t, lse, ent, g, g)
        assert torch.isfinite(dZ).all() and (dZ[0] == 0).all()
        assert (dZ[torch.isneginf(Z) & (torch.arange(V).cuda()[None] != t[:, None])] == 0).all()


def test_lowest_finite_values(F):
    """Masks made of the type's lowest value rather than -inf."""
    for dt in DT.values():
        Z = torch.randn(4, 3000).to(dt).cuda()
        Z[:, 10:2000] = torch.finfo(dt).min
        Z[3] = torch.finfo(dt).min
        t = torch.tensor([5, -1, 2500, 7]).cuda()
        lse, ent, _, _ = check(F, Z, t, 5)
        assert abs(float(ent[3]) - math.log(3000)) < 1e-3
        dZ = F.token_logprobs_bwd(Z, t, lse, ent, torch.ones(4).cuda(), torch.ones(4).cuda())
        assert torch.isfinite(dZ).all()


def test_domain_errors(F):
    for bad in (float("nan"), float("inf")):
        for T in (3, 600):
            Z = logits(T, 5000, "bf16", 1)
            Z[1, 3333] = bad
            ws = F.workspace(F.token_logprobs_workspace_size(T, 5000, 3))
            t = torch.zeros(T, dtype=torch.int64).cuda()
            logp, ent, lse, _, _ = F.token_logprobs(Z, t, 3, ws=ws)
            assert F.check_flags(ws) == F.ERR_DOMAIN
            keep = [i for i in range(T) if i != 1]
            assert torch.isfinite(logp[keep]).all() and torch.isfinite(lse[keep]).all()
    Z = logits(3, 100, "f32", 1)
    ws = F.workspace(F.token_logprobs_workspace_size(3, 100, 0))
    logp = F.token_logprobs(Z, torch.tensor([3, 100, -5]).cuda(), ws=ws)[0]
    assert F.check_flags(ws) == F.ERR_DOMAIN and logp[1] == 0 and logp[2] == 0
    F.token_logprobs(Z, torch.tensor([3, 99, -5]).cuda(), ws=ws)
    assert F.check_flags(ws) == F.OK


def test_gradient_against_differences(F):
    """Central differences in fp32: with a step of 1e-2 the third-order term is below 1e-4 of the derivative."""
    T, V = 5, 700
    Z, t = logits(T, V, "f32", 21, 1.0), targets(T, V, 3)
    g, h = torch.randn(T).cuda(), torch.randn(T).cuda()

    def loss(z):
        logp, ent, _, _, _ = F.token_logprobs(z, t)
        return float((logp.double() * g.double() + ent.double() * h.double()).sum())

    _, ent, lse, _, _ = F.token_logprobs(Z, t)
    dZ = F.token_logprobs_bwd(Z, t, lse, ent, g, h)
    for _ in range(4):
        d = dZ / dZ.norm() + 0.3 * torch.randn_like(Z) / Z.numel() ** 0.5
        e = 3e-2
        diff = (loss(Z + e * d) - loss(Z - e * d)) / (2 * e)
        assert abs(diff - float((dZ * d).sum())) <= 2e-3 * float(dZ.norm() * d.norm())


def test_in_place_repeatable_and_other_stream(F):
    Z, t = logits(700, 3001, "bf16", 5), targets(700, 3001, 6)
    a = F.token_logprobs(Z, t, 9)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        b = F.token_logprobs(Z, t, 9)
    s.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    g = torch.full((700,), -1.0 / 700).cuda()
    dZ = F.token_logprobs_bwd(Z, t, a[2], d_logp=g)
    Z2 = Z.clone()
    assert torch.equal(F.token_logprobs_bwd(Z2, t, a[2], d_logp=g, out=Z2), dZ)


def test_offsets_past_32_bits(F):
    """A tensor of more than 2^32 bytes: its last rows are those of a small copy."""
    T, V = 33000, 66000
    Z = torch.zeros(T, V, dtype=torch.bfloat16, device="cuda")
    Z[-3:] = logits(3, V, "bf16", 8)
    t = torch.full((T,), 7, device="cuda")
    logp, ent, lse, tl, ti = F.token_logprobs(Z, t, 4)
    small = Z[-3:].repeat(200, 1)  # as many rows that each is one workgroup's there too
    want = F.token_logprobs(small, t[:600], 4)
    for got, ref in zip((logp, ent, lse, tl, ti), want):
        assert torch.equal(got[-3:], ref[:3])
    g = torch.ones(T, device="cuda")
    dZ = F.token_logprobs_bwd(Z, t, lse, d_logp=g)
    assert torch.equal(dZ[-3:], F.token_logprobs_bwd(small, t[:600], want[2], d_logp=g[:600])[:3])


def test_refusals(F):
    Z = torch.randn(4, 100).cuda()
    t = torch.zeros(4, dtype=torch.int64).cuda()
    for call, status in ((lambda: F.token_logprobs(Z, t, 65), F.ERR_CONFIG), (lambda: F.token_logprobs(Z, t, -1), F.ERR_CONFIG),
                         (lambda: F.token_logprobs_bwd(Z, t, torch.zeros(4).cuda()), F.ERR_NULL),
                         (lambda: F.token_logprobs_bwd(Z, t, torch.zeros(4).cuda(), d_entropy=torch.zeros(4).cuda()), F.ERR_NULL),
                         (lambda: F.token_logprobs_bwd(Z, None, torch.zeros(4).cuda(), d_logp=torch.zeros(4).cuda()), F.ERR_NULL),
                         (lambda: F.token_logprobs(torch.empty(4, 0).cuda(), None), F.ERR_SHAPE)):
        with pytest.raises(F.FocusError) as e:
            call()
        assert e.value.status == status
    with pytest.raises(ValueError):
        F.token_logprobs(Z, t.int())
    with pytest.raises(ValueError):
        F.token_logprobs(Z, t[:3])
    with pytest.raises(ValueError):
        F.token_logprobs(Z.t(), torch.zeros(100, dtype=torch.int64).cuda())
    with pytest.raises(TypeError):
        F.token_logprobs(Z.half(), t)
    assert F.token_logprobs(torch.empty(0, 100).cuda(), None)[1].shape == (0,)


def test_more_rows_than_one_launch_holds(F):
    """The rows past 2^23 - 1 (forward) and 2^24 - 1 (gradient) against calls of their own."""
    T, V, tail = (1 << 24) + 1000, 5, 1500
    Z = torch.randn(T, V, device="cuda", generator=torch.Generator("cuda").manual_seed(4)).bfloat16()
    target = (torch.arange(T, device="cuda") * 7) % (V + 1) - 1
    some, mine = Z[-tail:].contiguous(), target[-tail:].contiguous()
    got, ref = F.token_logprobs(Z, target, 2), F.token_logprobs(some, mine, 2)
    for a, b in zip(got, ref):
        assert torch.equal(a[-tail:], b)
    g = torch.linspace(-1, 1, T, device="cuda")
    dZ = F.token_logprobs_bwd(Z, target, got[2], got[1], g, g)
    assert torch.equal(dZ[-tail:], F.token_logprobs_bwd(some, mine, ref[2], ref[1], g[-tail:].contiguous(), g[-tail:].contiguous()))


def test_refuses_tensors_of_the_host(F):
    Z, t = torch.zeros(3, 16, device="cuda"), torch.zeros(3, dtype=torch.int64, device="cuda")
    logp, entropy, lse, _, _ = F.token_logprobs(Z, t)
    for call in (lambda: F.token_logprobs(Z.cpu(), t), lambda: F.token_logprobs(Z, t.cpu()),
                 lambda: F.token_logprobs_bwd(Z, t, lse.cpu(), d_logp=lse), lambda: F.token_logprobs_bwd(Z, t, lse, d_logp=lse.cpu())):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("top", [1, 5, 64])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_rows_in_parts(F, dt, top):
    """Few long rows: the largest in one part or in all, equal over the parts, a part without a token, a row without any."""
    g = torch.Generator().manual_seed(8)
    for V in (65537, 100003, 262144):
        i = torch.arange(V)
        rows = [torch.randn(V, generator=g), torch.zeros(V), i.float() / 64, -i.float() / 64, torch.where(i > V - 70, 3.0, -1.0),
                torch.where(i % 15000 == 0, 4.0, torch.randn(V, generator=g)), torch.where(i < 40000, -math.inf, 1.0),
                torch.where(i == V - 1, 0.0, -math.inf), torch.full((V,), -math.inf),
                torch.full((V,), torch.finfo(DT[dt]).min)]
        Z = torch.stack(rows).to(DT[dt]).cuda()
        announce(f"rows in parts {dt} V={V} top={top}")
        t = targets(len(rows), V, 4)
        lse, ent, lp, none = check(F, Z, t, top)
        assert none.tolist() == [False] * 8 + [True, False] and ent[8] == 0
        for n in (1, 3, 9):  # other numbers of rows are other numbers of parts
            check(F, Z[:n].contiguous(), t[:n].contiguous(), top)


def test_many_rows_in_parts(F):
    Z, t = logits(64, 300001, "bf16", 12), targets(64, 300001, 3)
    check(F, Z, t, 6)
    check(F, Z[:63], t[:63].contiguous(), 6)


def test_domain_errors_of_parts(F):
    for bad in (float("nan"), float("inf")):
        Z = logits(5, 90000, "bf16", 1)
        Z[1, 88888] = bad
        ws = F.workspace(F.token_logprobs_workspace_size(5, 90000, 3))
        logp, _, lse, _, _ = F.token_logprobs(Z, torch.zeros(5, dtype=torch.int64).cuda(), 3, ws=ws)
        assert F.check_flags(ws) == F.ERR_DOMAIN
        assert torch.isfinite(logp[[0, 2, 3, 4]]).all() and torch.isfinite(lse[[0, 2, 3, 4]]).all()
    Z[1, 88888] = 0.0
    logp = F.token_logprobs(Z, torch.tensor([3, 90000, -5, 0, 1]).cuda(), ws=ws)[0]
    assert F.check_flags(ws) == F.ERR_DOMAIN and logp[1] == 0 and logp[2] == 0
