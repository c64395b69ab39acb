"""GPU tests of focus_linear_ce_fwd / focus_linear_ce_bwd against the definition in float64.

Bounds. A logit is a sum of K fp32 products: independent roundings of partial sums no larger than S = max(1, max |z|) make it off
by 4 sqrt(K) 2^-24 S; that, and the rounding of lse itself (2 x 2^-24 |lse|) and of the sum of exponentials (2^-20), bounds
lse and logp. Gradients: p is off by what z and lse are, relative to itself, in fp32. With bf16 operands D is rounded to bf16
relative to the token's larger factor, once, and X scaled by that factor, once: a term of a sum is off by 2 x 2^-8 at most,
and the result by half a step, 2^-8. Those roundings are independent, so that the whole gradient is held to 3 roundings'
root mean square, sqrt(3) 2^-8 / sqrt(3) = 3.9e-3 of its norm. fp32: 1e-5 of the norm, sums of up to 10^4 terms.
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


def make(T, V, K, dt, seed, ignored=0.2, spread=2.0):
    g = torch.Generator().manual_seed(seed)
    W = (torch.randn(V, K, generator=g) * spread / math.sqrt(K)).to(dt)
    target = torch.randint(0, V, (T,), generator=g)
    X = torch.randn(T, K, generator=g)
    if spread > 0:  # the target's logit is raised by up to 8
        X = X + 8.0 * torch.rand(T, 1, generator=g) / spread ** 2 * W.float()[target]
    target[torch.rand(T, generator=g) < ignored] = -1
    d_logp = -(0.2 + torch.rand(T, generator=g)) / max(1, T)
    d_lse = 0.1 * torch.randn(T, generator=g) / max(1, T)
    return [t.cuda() for t in (X.to(dt), W, target, d_logp, d_lse)]


def reference(X, W, target, g, h):
    """logp, lse, D, dX, dW in float64 and the largest logit's size."""
    x, w = X.double(), W.double()
    z = x @ w.t()
    lse = torch.logsumexp(z, 1)
    kept = torch.nonzero(target >= 0)[:, 0]
    logp = torch.zeros_like(lse)
    logp[kept] = z[kept, target[kept]] - lse[kept]
    gk = torch.zeros_like(lse)
    if g is not None:
        gk[kept] = g.double()[kept]
    hk = torch.zeros_like(lse) if h is None else h.double()
    D = (hk - gk)[:, None] * (z - lse[:, None]).exp()
    D[kept, target[kept]] += gk[kept]
    return logp, lse, D, D @ w, D.t() @ x, max(1.0, float(z.abs().max()))


def z_error(K, S):
    return 4.0 * math.sqrt(K) * 2.0 ** -24 * S


def check(F, X, W, target, g, h, dw_dtype=None, ws=None):
    K = X.shape[1]
    logp, lse = F.linear_ce_fwd(X, W, target, ws=ws)
    dX, dW = F.linear_ce_bwd(X, W, target, lse, g, h, dw_dtype=dw_dtype, ws=ws)
    torch.cuda.synchronize()
    rlogp, rlse, D, rdX, rdW, S = reference(X, W, target, g, h)
    lim = z_error(K, S) + 2.0 ** -20
    assert ((lse.double() - rlse).abs() <= lim + 2.0 ** -23 * rlse.abs()).all(), float((lse.double() - rlse).abs().max())
    assert ((logp.double() - rlogp).abs() <= 2 * lim + 2.0 ** -23 * rlogp.abs()).all(), float((logp.double() - rlogp).abs().max())
    assert (logp[target < 0] == 0).all()
    bf16 = X.dtype == torch.bfloat16
    p_err = 2 * (lim + 2.0 ** -23 * float(rlse.abs().max()))
    for got, ref, mags, what in ((dX, rdX, D.abs() @ W.double().abs(), "dX"), (dW, rdW, D.abs().t() @ X.double().abs(), "dW")):
        step = 2.0 ** -8 if got.dtype == torch.bfloat16 else 2.0 ** -24
        terms = (2 * 2.0 ** -8 if bf16 else 0.0) + p_err + 1e-5
        err = (got.double() - ref).abs()
        assert (err <= terms * mags + step * ref.abs() + 1e-30).all(), (what, float(err.max()), float(ref.abs().max()))
        size = float(ref.norm())
        assert float(err.norm()) <= (3.9e-3 if bf16 else 1e-5 + p_err) * size + 1e-30, (what, float(err.norm()) / size)
    return logp, lse, dX, dW


SHAPES = [(1, 1, 1), (1, 3, 8), (3, 1000, 16), (1, 4099, 256), (7, 257, 100), (64, 512, 64), (129, 511, 80), (300, 5003, 1008),
          (33, 777, 33), (257, 1024, 128), (513, 300, 320), (1000, 2049, 48), (17, 20001, 96), (2, 2, 4096)]


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("T,V,K", SHAPES)
def test_against_definition(F, T, V, K, dt):
    announce(f"linear ce {dt} T={T} V={V} K={K}")
    X, W, target, g, h = make(T, V, K, DT[dt], T * 7 + V + K)
    ws = F.workspace(F.linear_ce_workspace_size(T, V, K))
    ws[256:] = 255  # NaN: nothing is read before it is written
    check(F, X, W, target, g, h, ws=ws)
    assert F.check_flags(ws) == F.OK


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_uniform_weights_of_the_tokens(F, dt):
    # the mean over the tokens that count, whose weight is no power of two: it must not be rounded into every term alike
    announce(f"linear ce mean {dt}")
    X, W, target, g, _ = make(700, 3000, 256, DT[dt], 21)
    n = int((target >= 0).sum())
    logp, lse, dX, dW = check(F, X, W, target, torch.full_like(g, -1.0 / n), None)
    _, _, _, rdX, rdW, _ = reference(X, W, target, torch.full_like(g, -1.0 / n), None)
    for got, ref in ((dX, rdX), (dW, rdW)):
        along = float((got.double() * ref).sum() / ref.square().sum())
        assert abs(along - 1.0) <= (5e-4 if dt == "bf16" else 1e-5), along


def test_fp32_weight_gradient_of_bf16_operands(F):
    announce("linear ce fp32 dW")
    X, W, target, g, h = make(300, 900, 160, torch.bfloat16, 22)
    _, lse, _, dW = check(F, X, W, target, g, h, dw_dtype=torch.float32)
    _, half = F.linear_ce_bwd(X, W, target, lse, g, h)
    assert dW.dtype == torch.float32 and half.dtype == torch.bfloat16
    assert torch.equal(dW.bfloat16(), half)


@pytest.mark.parametrize("T,K", [(5, 33), (300, 1), (300, 1001)])
def test_padded_rows(F, T, K):
    # the workspace holds NaN, and the bytes around the outputs stay as they are
    announce(f"linear ce padded T={T} K={K}")
    X, W, target, g, h = make(T, 901, K, torch.bfloat16, 33)
    ws = F.workspace(F.linear_ce_workspace_size(T, 901, K))
    ws[256:] = 255
    _, lse, dX, dW = check(F, X, W, target, g, h, dw_dtype=torch.float32, ws=ws)
    rows = lambda n, dt: torch.full((n * K + 64,), 7.0, dtype=dt, device="cuda")
    x, w = rows(T, torch.bfloat16), rows(901, torch.bfloat16)
    a, b = F.linear_ce_bwd(X, W, target, lse, g, h, ws=ws, out=x[:T * K].view(T, K), dw_out=w[:901 * K].view(901, K))
    assert torch.equal(a, dX) and torch.equal(b, dW.bfloat16())
    assert (x[T * K:] == 7).all() and (w[901 * K:] == 7).all()
    assert torch.equal(F.linear_ce_bwd(X, W, target, lse, g, h, want_dw=False, ws=ws)[0], dX)
    assert torch.equal(F.linear_ce_bwd(X, W, target, lse, g, h, want_dx=False, dw_dtype=torch.float32, ws=ws)[1], dW)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_one_gradient_at_a_time(F, dt):
    announce(f"linear ce parts {dt}")
    X, W, target, g, h = make(150, 700, 64, DT[dt], 23)
    _, lse = F.linear_ce_fwd(X, W, target)
    dX, dW = F.linear_ce_bwd(X, W, target, lse, g, h)
    a, none = F.linear_ce_bwd(X, W, target, lse, g, h, want_dw=False)
    assert none is None and torch.equal(a, dX)
    none, b = F.linear_ce_bwd(X, W, target, lse, g, h, want_dx=False)
    assert none is None and torch.equal(b, dW)
    check(F, X, W, target, g, None)
    check(F, X, W, target, None, h)
    assert torch.equal(F.linear_ce_fwd(X, W)[1], lse) and F.linear_ce_fwd(X, W)[0] is None
    none_kept = torch.full_like(target, -100)
    logp, _ = F.linear_ce_fwd(X, W, none_kept)
    dX, dW = F.linear_ce_bwd(X, W, none_kept, lse, g)
    assert not logp.any() and not dX.any() and not dW.any()
    without_target, _ = F.linear_ce_bwd(X, W, None, lse, d_lse=h)
    ref = reference(X, W, none_kept, None, h)[3]
    assert float((without_target.double() - ref).norm() / ref.norm()) <= (3.9e-3 if dt == "bf16" else 1e-5)


def test_one_token_many_times_and_one_target(F):
    announce("linear ce repeated")
    X, W, target, g, h = make(400, 600, 64, torch.bfloat16, 24, ignored=0.0)
    target.fill_(599)
    X[:] = X[0]
    check(F, X, W, target, g, h)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_logits_of_many_sizes(F, dt):
    announce(f"linear ce sizes {dt}")
    for spread in (0.0, 0.01, 30.0):
        X, W, target, g, h = make(130, 777, 128, DT[dt], 25, spread=spread)
        check(F, X, W, target, g, h)


def test_gradients_against_differences(F):
    announce("linear ce differences")
    X, W, target, g, h = make(20, 50, 24, torch.float32, 26)
    _, lse = F.linear_ce_fwd(X, W, target)
    dX, dW = F.linear_ce_bwd(X, W, target, lse, g, h)
    f = lambda x, w: float((reference(x, w, target, g, h)[0] * g.double()).sum() + (reference(x, w, target, g, h)[1] * h.double()).sum())
    gen = torch.Generator(device="cuda").manual_seed(5)
    for which, got in ((0, dX), (1, dW)):
        at = [X.double(), W.double()]
        step = torch.randn(at[which].shape, generator=gen, device="cuda", dtype=torch.float64)
        v = []
        for s in (1e-5, -1e-5):
            c = list(at)
            c[which] = c[which] + s * step
            v.append(f(*c))
        terms = got.double() * step
        assert abs(float(terms.sum()) - (v[0] - v[1]) / 2e-5) <= 2e-5 * float(terms.abs().sum()) + 1e-8


def test_bad_targets_and_logits_raise_the_flag(F):
    announce("linear ce flags")
    X, W, target, g, _ = make(40, 300, 64, torch.bfloat16, 27)
    ws = F.workspace(F.linear_ce_workspace_size(40, 300, 64))
    target[3] = 300
    logp, lse = F.linear_ce_fwd(X, W, target, ws=ws)
    assert F.check_flags(ws) == F.ERR_DOMAIN and logp[3] == 0
    F.linear_ce_bwd(X, W, target, lse, g, ws=ws)
    assert F.check_flags(ws) == F.ERR_DOMAIN
    target[3] = 2 ** 40
    F.linear_ce_fwd(X, W, target, ws=ws)
    assert F.check_flags(ws) == F.ERR_DOMAIN
    target[3] = -2 ** 40
    logp, lse = F.linear_ce_fwd(X, W, target, ws=ws)
    F.linear_ce_bwd(X, W, target, lse, g, ws=ws)
    assert F.check_flags(ws) == F.OK and logp[3] == 0
    for bad in (math.nan, math.inf, -math.inf):
        Y = X.clone()
        Y[7, 3] = bad
        a, _ = F.linear_ce_fwd(Y, W, target, ws=ws)
        assert F.check_flags(ws) == F.ERR_DOMAIN
        keep = torch.arange(40, device="cuda") != 7
        assert torch.equal(a[keep], logp[keep])  # the other tokens are not touched by it
    lse[5] = 1e6
    g[5] = -1.0
    target[5] = 1
    F.linear_ce_bwd(X, W, target, lse, g, ws=ws)
    assert F.check_flags(ws) == F.ERR_DOMAIN


@pytest.mark.parametrize("dt,K", [("bf16", 64), ("bf16", 24), ("f32", 64), ("f32", 24)])
def test_tokens_without_a_gradient_may_hold_anything(F, dt, K):
    announce(f"linear ce padding {dt} K={K}")
    X, W, target, g, _ = make(300, 700, K, DT[dt], 29)
    ws = F.workspace(F.linear_ce_workspace_size(300, 700, K))
    logp, lse = F.linear_ce_fwd(X, W, target, ws=ws)
    g[10:14] = 0.0
    out = target < 0
    out[10:14] = True
    want = F.linear_ce_bwd(X, W, target, lse, g, ws=ws)
    bad = torch.tensor([math.nan, math.inf, -math.inf], device="cuda", dtype=X.dtype)
    Y, at = X.clone(), torch.nonzero(out)[:, 0]
    Y[at] = bad[at % 3][:, None]
    Z = torch.where((target < 0)[:, None], Y, X)
    a, rest = F.linear_ce_fwd(Z, W, target, ws=ws)
    assert F.check_flags(ws) == F.OK and torch.equal(a, logp) and torch.equal(rest[target >= 0], lse[target >= 0])
    lse[out] = math.nan
    got = F.linear_ce_bwd(Y, W, target, lse, g, ws=ws)
    assert F.check_flags(ws) == F.OK and all(torch.equal(x, y) for x, y in zip(got, want))
    assert not got[0][out].any()
    F.linear_ce_fwd(Z, W, None, ws=ws)  # every token counts
    assert F.check_flags(ws) == F.ERR_DOMAIN


def test_gradients_smaller_than_the_normal_numbers(F):
    # fp32 results below 2^-126 have steps of 2^-149, bf16 ones of 2^-133; apart from that the bounds are those of any size
    announce("linear ce tiny")
    X, W, target, _, _ = make(200, 300, 64, torch.bfloat16, 30)
    g = -(1.0 + torch.rand(200, generator=torch.Generator().manual_seed(31)).cuda()) * 2.0 ** -127
    _, lse = F.linear_ce_fwd(X, W, target)
    dX, dW = F.linear_ce_bwd(X, W, target, lse, g, dw_dtype=torch.float32)
    _, rlse, D, rdX, rdW, S = reference(X, W, target, g, None)
    terms = 2 * 2.0 ** -8 + 2 * (z_error(64, S) + 2.0 ** -20 + 2.0 ** -23 * float(rlse.abs().max())) + 1e-5
    for got, ref, mags, step in ((dX, rdX, D.abs() @ W.double().abs(), 2.0 ** -133), (dW, rdW, D.abs().t() @ X.double().abs(), 2.0 ** -149)):
        err = (got.double() - ref).abs()
        assert (err <= terms * mags + 2.0 ** -8 * ref.abs() + step).all(), float(err.max())


@pytest.mark.parametrize("dt,T,K", [("bf16", 4, 32), ("bf16", 20, 32), ("bf16", 600, 32), ("bf16", 20, 24), ("f32", 20, 32), ("f32", 20, 24)])
def test_the_largest_logits(F, dt, T, K):
    # one product each, so that logits are exact; neighbours differ by 2^15 and more, so that lse is the largest
    announce(f"linear ce largest {dt} T={T} K={K}")
    g = torch.Generator().manual_seed(32)
    X = torch.zeros(T, K)
    X[:, 0] = 2.0 ** 15
    W = torch.zeros(500, K)
    W[:, 0] = torch.randint(-127, 128, (500,), generator=g) * 2.0 ** 7
    W[77, 0] = 2.0 ** 14
    target = torch.randint(0, 500, (T,), generator=g)
    ws = F.workspace(F.linear_ce_workspace_size(T, 500, K))
    for sign in (1.0, -1.0):  # the other sign: the least logit in size is the largest
        x, w = (sign * X).to(DT[dt]).cuda(), W.to(DT[dt]).cuda()
        z = (x.double() @ w.double().t())
        logp, lse = F.linear_ce_fwd(x, w, target.cuda(), ws=ws)
        m = z.max(1).values
        assert F.check_flags(ws) == F.OK
        assert ((lse.double() - m).abs() <= 2.0 + 2.0 ** -24 * m.abs()).all()
        assert ((logp.double() - (z.gather(1, target.cuda()[:, None])[:, 0] - m)).abs() <= 2.0 + 2.0 ** -22 * m.abs()).all()
    F.linear_ce_fwd(2.0 * X.to(DT[dt]).cuda(), w, target.cuda(), ws=ws)
    assert F.check_flags(ws) == F.ERR_DOMAIN


def test_pieces_of_the_vocabulary(F):
    # tokens enough that the vocabulary takes several pieces, the last one odd
    T, V, K = 40000, 21013, 32
    announce("linear ce pieces")
    g = torch.Generator(device="cuda").manual_seed(3)
    X = torch.randn(T, K, generator=g, device="cuda").bfloat16()
    W = (0.3 * torch.randn(V, K, generator=g, device="cuda")).bfloat16()
    target = torch.randint(0, V, (T,), generator=g, device="cuda")
    w = torch.full((T,), -1.0 / T, device="cuda")
    logp, lse = F.linear_ce_fwd(X, W, target)
    dX, dW = F.linear_ce_bwd(X, W, target, lse, w)
    rdW = torch.zeros(V, K, dtype=torch.float64, device="cuda")
    for r in range(0, T, 8000):
        e = slice(r, r + 8000)
        rlogp, rlse, _, rdX, part, S = reference(X[e], W, target[e], w[e], None)
        rdW += part
        assert ((lse[e].double() - rlse).abs() <= z_error(K, S) + 2.0 ** -20 + 2.0 ** -23 * rlse.abs()).all()
        assert float((dX[e].double() - rdX).norm() / rdX.norm()) <= 3.9e-3
    assert float((dW.double() - rdW).norm() / rdW.norm()) <= 3.9e-3


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_the_same_bits_twice_and_with_more_workspace(F, dt):
    announce(f"linear ce determinism {dt}")
    X, W, target, g, h = make(333, 2500, 160, DT[dt], 28)
    a = check(F, X, W, target, g, h)
    ws = F.workspace(2 * F.linear_ce_workspace_size(1000, 2500, 160))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        logp, lse = F.linear_ce_fwd(X, W, target, ws=ws)
        b = (logp, lse) + F.linear_ce_bwd(X, W, target, lse, g, h, ws=ws)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_nothing_to_do(F):
    X, W, target, g, h = make(0, 30, 16, torch.bfloat16, 1)
    logp, lse = F.linear_ce_fwd(X, W, target)
    dX, dW = F.linear_ce_bwd(X, W, target, lse, g, h)
    assert logp.shape == lse.shape == (0,) and dX.shape == (0, 16) and dW.shape == (30, 16) and not dW.any()


def test_refusals(F):
    X, W, target, g, h = make(8, 64, 32, torch.bfloat16, 2)
    _, lse = F.linear_ce_fwd(X, W, target)
    for bad in (lambda: F.linear_ce_fwd(X, W.float(), target), lambda: F.linear_ce_fwd(X[:, :16].contiguous(), W, target),
                lambda: F.linear_ce_fwd(X, W, target.int()), lambda: F.linear_ce_fwd(X, W.t(), target),
                lambda: F.linear_ce_fwd(X.cpu(), W, target), lambda: F.linear_ce_bwd(X, W, target, lse.double(), g),
                lambda: F.linear_ce_bwd(X, W, target, lse, g, out=X.float()), lambda: F.linear_ce_bwd(X, W, target, lse, g, dw_out=X)):
        with pytest.raises((ValueError, TypeError)):
            bad()
    for status, bad in ((F.ERR_NULL, lambda: F.linear_ce_bwd(X, W, target, lse)),
                        (F.ERR_NULL, lambda: F.linear_ce_bwd(X, W, None, lse, g)),
                        (F.ERR_NULL, lambda: F.linear_ce_bwd(X, W, target, lse, g, want_dx=False, want_dw=False)),
                        (F.ERR_SHAPE, lambda: F.linear_ce_bwd(X, W, target, lse, g, out=X)),
                        (F.ERR_SHAPE, lambda: F.linear_ce_bwd(X, W, target, lse, g, dw_out=W)),
                        (F.ERR_DTYPE, lambda: F.linear_ce_bwd(X.float(), W.float(), target, lse, g, dw_dtype=torch.bfloat16)),
                        (F.ERR_WORKSPACE, lambda: F.linear_ce_fwd(X, W, target, ws=F.workspace(256)))):
        with pytest.raises(F.FocusError) as e:
            bad()
        assert e.value.status == status
