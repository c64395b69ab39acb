"""GPU tests of focus_attention_fwd / focus_attention_bwd against the definition in float64.

Bounds, with u = 2^-9 the relative rounding error of bf16 and every sum in fp32:
  O: each probability is rounded once, so |dO_err| <= u sum P|v|, then the result once, u |O|;
  dv: u sum P|dO| + u |dv|;
  dS: the rounding of dS, u |dS|, and the error of delta = rowsum(dO O) from the rounded O, sum |dO| |O_err|, times P;
  dq, dk: scale sum |dS_err| |k| (|q|) + u |dq|.
They are evaluated from the reference's own matrices and doubled, which leaves room for the fp32 sums and the exponentials
(about 1e-5). In fp32 u is 2^-24, the same expressions are taken 32 times (sums of up to a few hundred terms, scores of
size 30 whose rounding enters the exponent: 30 x 2^-24 x 1.44).
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


def ends(lengths):
    out = [0]
    for n in lengths:
        out.append(out[-1] + n)
    return out


def make(lq, lk, Hq, Hkv, D, dt, seed, scale=1.3):
    g = torch.Generator().manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g)
    tq, tk = sum(lq), sum(lk)
    return {"q": (rnd(tq, Hq, D) * scale).to(dt).cuda(), "k": rnd(tk, Hkv, D).to(dt).cuda(), "v": rnd(tk, Hkv, D).to(dt).cuda(),
            "dO": rnd(tq, Hq, D).to(dt).cuda()}


def reference(t, lq, lk, causal, scale, u):
    """Results in float64 and the bounds of their errors."""
    q, k, v, G = (t[n].double().cpu() for n in ("q", "k", "v", "dO"))
    Hq, Hkv = q.shape[1], k.shape[1]
    r = {"O": torch.zeros_like(q), "lse": torch.full((Hq, q.shape[0]), -math.inf, dtype=torch.float64), "dq": torch.zeros_like(q),
         "dk": torch.zeros_like(k), "dv": torch.zeros_like(v)}
    e = {n: torch.zeros_like(x) for n, x in r.items() if n != "lse"}
    eq, ek = ends(lq), ends(lk)
    for s in range(len(lq)):
        a, b = slice(eq[s], eq[s + 1]), slice(ek[s], ek[s + 1])
        for h in range(Hq):
            hk = h // (Hq // Hkv)
            Q, K, V, g = q[a, h], k[b, hk], v[b, hk], G[a, h]
            if lq[s] == 0 or lk[s] == 0:
                continue
            S = Q @ K.T * scale
            if causal:
                S = S.masked_fill(~torch.ones(lq[s], lk[s], dtype=torch.bool).tril(lk[s] - lq[s]), -math.inf)
            m = S.amax(1, keepdim=True)
            some = m > -math.inf
            P = torch.where(some, (S - torch.where(some, m, 0.0)).exp(), 0.0)
            l = P.sum(1, keepdim=True)
            P = torch.where(some, P / torch.where(some, l, 1.0), 0.0)
            O = P @ V
            r["O"][a, h] = O
            r["lse"][h, a] = torch.where(some, m + l.clamp(min=1e-300).log(), -math.inf)[:, 0]
            eO = u * (P @ V.abs()) + u * O.abs()
            e["O"][a, h] = eO
            delta = (g * O).sum(1, keepdim=True)
            dS = P * (g @ V.T - delta)
            eS = u * dS.abs() + P * (g.abs() * eO).sum(1, keepdim=True) + u * P * (g.abs() @ V.abs().T) * (u < 1e-6)
            r["dq"][a, h] = dS @ K * scale
            r["dk"][b, hk] += dS.T @ Q * scale
            r["dv"][b, hk] += P.T @ g
            e["dq"][a, h] = abs(scale) * (eS @ K.abs())
            e["dk"][b, hk] += abs(scale) * (eS.T @ Q.abs())
            e["dv"][b, hk] += u * (P.T @ g.abs())
    for n in ("dq", "dk", "dv"):
        e[n] += u * r[n].abs()
    return r, e


def check(got, ref, err, name, times):
    got = got.double().cpu()
    lim = times * err + 1e-6 * ref.abs().max().clamp(min=1e-3) * (1 if times > 4 else 10)
    bad = ~((got - ref).abs() <= lim)
    assert not bad.any(), (name, int(bad.sum()), float(((got - ref).abs() / lim).nan_to_num(1e9).max()))


def run_case(F, lq, lk, Hq, Hkv, D, dt, causal, seed=0, scale=None, single=False):
    announce(f"attention {dt} lq={lq} lk={lk} heads={Hq}/{Hkv} D={D} causal={causal}")
    t = make(lq, lk, Hq, Hkv, D, DT[dt], seed)
    cq = ck = None
    if not single:
        cq = torch.tensor(ends(lq), dtype=torch.int32).cuda()
        ck = torch.tensor(ends(lk), dtype=torch.int32).cuda() if lk is not lq else None
    ws = F.workspace(F.attention_workspace_size(t["q"], t["k"], len(lq)))
    O, lse = F.attention_fwd(t["q"], t["k"], t["v"], cq, ck, causal, scale, ws=ws)
    dq, dk, dv = F.attention_bwd(t["dO"], t["q"], t["k"], t["v"], O, lse, cq, ck, causal, scale, ws=ws)
    torch.cuda.synchronize()
    assert F.check_flags(ws) == F.OK
    u, times = (2.0 ** -9, 2.0) if dt == "bf16" else (2.0 ** -24, 32.0)
    r, e = reference(t, lq, lk, causal, D ** -0.5 if scale is None else scale, u)
    check(O, r["O"], e["O"], "O", times)
    none = r["lse"] == -math.inf
    assert torch.equal(torch.isneginf(lse.cpu()), none)
    assert ((lse.double().cpu() - r["lse"])[~none].abs() <= 2e-5 * (1 + r["lse"][~none].abs())).all()
    check(dq, r["dq"], e["dq"], "dq", times)
    check(dk, r["dk"], e["dk"], "dk", times)
    check(dv, r["dv"], e["dv"], "dv", times)


LENGTHS = [[1], [2, 1, 3], [31, 32, 33], [64, 65, 127, 128, 129], [257], [0, 5, 0, 0, 70, 0], [1] * 70]


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lengths", LENGTHS, ids=lambda v: "-".join(map(str, v[:6])))
def test_self_attention(F, lengths, causal, dt):
    run_case(F, lengths, lengths, 4, 2, 64, dt, causal)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("D", [8, 16, 24, 32, 40, 72, 80, 96, 104, 128])
def test_head_dims(F, D, dt):
    run_case(F, [70, 9], [70, 9], 3, 1, D, dt, True, seed=D)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (8, 1), (8, 8), (6, 2), (16, 2)])
def test_head_layouts(F, Hq, Hkv, dt):
    run_case(F, [45, 130], [45, 130], Hq, Hkv, 128, dt, True, seed=Hq)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lq,lk", [([1], [300]), ([1, 1, 1], [1, 64, 129]), ([5, 40], [100, 41]), ([30, 0, 7], [10, 20, 0]),
                                   ([64], [1]), ([150], [20]), ([3], [2000])], ids=str)
def test_queries_and_keys_of_different_lengths(F, lq, lk, causal, dt):
    """Queries that are the end of longer keys; and causal queries before the first key, whose rows are empty."""
    run_case(F, lq, lk, 4, 2, 128, dt, causal, seed=sum(lk))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_one_sequence_without_ends(F, dt):
    run_case(F, [333], [333], 2, 2, 128, dt, True, single=True)
    run_case(F, [17], [333], 2, 1, 128, dt, True, single=True)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_scale(F, dt):
    run_case(F, [50], [50], 2, 1, 64, dt, True, scale=0.02)
    run_case(F, [50], [50], 2, 1, 64, dt, True, scale=0.0)
    run_case(F, [50], [50], 2, 1, 64, dt, True, scale=-0.1)


def test_longer_sequences(F):
    run_case(F, [1500, 600], [1500, 600], 4, 1, 128, "bf16", True)
    run_case(F, [700], [700], 2, 2, 64, "bf16", False)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_large_scores(F, dt):
    """Scores up to some 1e4: the softmax picks one key; no overflow, rows sum to one."""
    g = torch.Generator().manual_seed(1)
    q, k = (torch.randn(90, 2, 64, generator=g).to(DT[dt]).cuda() * 60 for _ in range(2))
    v = torch.ones(90, 2, 64).to(DT[dt]).cuda()
    O, lse = F.attention_fwd(q, k, v)
    assert torch.isfinite(lse).all() and (O.float() - 1.0).abs().max() <= 2.0 ** -7
    dq, dk, dv = F.attention_bwd(torch.ones_like(q), q, k, v, O, lse)
    assert all(torch.isfinite(x).all() for x in (dq, dk, dv))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_nothing_of_other_sequences(F, dt, bad):
    """Sequences 1 and 3 are full of `bad` in every input: the results of 0, 2 and 4 are bit for bit the same."""
    lengths = [70, 33, 129, 5, 64]
    e = ends(lengths)
    cu = torch.tensor(e, dtype=torch.int32).cuda()
    t = make(lengths, lengths, 4, 2, 128, DT[dt], 3)
    O, lse = F.attention_fwd(t["q"], t["k"], t["v"], cu)
    grads = F.attention_bwd(t["dO"], t["q"], t["k"], t["v"], O, lse, cu)
    x = {n: v.clone() for n, v in t.items()}
    for s in (1, 3):
        for v in x.values():
            v[e[s]:e[s + 1]] = bad
    O2, lse2 = F.attention_fwd(x["q"], x["k"], x["v"], cu)
    grads2 = F.attention_bwd(x["dO"], x["q"], x["k"], x["v"], O2, lse2, cu)
    for s in (0, 2, 4):
        r = slice(e[s], e[s + 1])
        assert torch.equal(O[r], O2[r]) and torch.equal(lse[:, r], lse2[:, r])
        for a, b in zip(grads, grads2):
            assert torch.equal(a[r], b[r])


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_nothing_of_hidden_keys(F, dt, bad):
    """NaN and infinities in the keys that a causal query does not see."""
    t = make([100], [100], 2, 1, 64, DT[dt], 4)
    O, lse = F.attention_fwd(t["q"], t["k"], t["v"])
    k = t["k"].clone()
    k[60:] = bad
    O2, lse2 = F.attention_fwd(t["q"], k, t["v"])
    assert torch.equal(O[:60], O2[:60]) and torch.equal(lse[:, :60], lse2[:, :60])


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("cu", [[10, 40, 90], [400, 430, 480], [700, 730, 780]], ids=str)
def test_rows_of_no_sequence_are_left_alone(F, dt, cu):
    """Rows before the first sequence, some of them whole tiles of queries or keys, and behind the last."""
    T, a, b = 800, cu[0], cu[-1]
    t = make([T], [T], 2, 2, 64, DT[dt], 6)
    cu = torch.tensor(cu, dtype=torch.int32).cuda()
    for v in t.values():
        v[:a] = float("nan")
        v[b:] = float("nan")
    O, lse = torch.full_like(t["q"], 7.0), torch.full((2, T), 7.0).cuda()
    F.attention_fwd(t["q"], t["k"], t["v"], cu, out=O, lse=lse)
    out = tuple(torch.full_like(t["q"], 7.0) for _ in range(3))
    F.attention_bwd(t["dO"], t["q"], t["k"], t["v"], O, lse, cu, out=out)
    for x in (O, lse.t(), *out):
        assert (x[:a] == 7.0).all() and (x[b:] == 7.0).all() and torch.isfinite(x[a:b]).all()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_slices_of_a_fused_product(F, dt):
    Hq, Hkv, D, lengths = 4, 2, 64, [50, 77]
    g = torch.Generator().manual_seed(8)
    T = sum(lengths)
    fused = torch.randn(T, (Hq + 2 * Hkv) * D + 16, generator=g).to(DT[dt]).cuda()
    cut = lambda x: (x[:, :Hq * D].unflatten(1, (Hq, D)), x[:, Hq * D:(Hq + Hkv) * D].unflatten(1, (Hkv, D)),
                     x[:, (Hq + Hkv) * D:(Hq + 2 * Hkv) * D].unflatten(1, (Hkv, D)))
    q, k, v = cut(fused)
    cu = torch.tensor(ends(lengths), dtype=torch.int32).cuda()
    O, lse = F.attention_fwd(q, k, v, cu)
    O2, lse2 = F.attention_fwd(q.contiguous(), k.contiguous(), v.contiguous(), cu)
    assert torch.equal(O, O2) and torch.equal(lse, lse2)
    dO = torch.randn(T, Hq, D, generator=g).to(DT[dt]).cuda()
    d = torch.full_like(fused, 7.0)
    F.attention_bwd(dO, q, k, v, O, lse, cu, out=cut(d))
    for a, b in zip(cut(d), F.attention_bwd(dO, q.contiguous(), k.contiguous(), v.contiguous(), O, lse, cu)):
        assert torch.equal(a, b)
    assert (d[:, -16:] == 7.0).all()


def test_gradient_against_differences(F):
    """Central differences of L = sum(O G) in fp32 along directions that hold the gradient: the third-order term with a
    step of 1e-2 and the rounding of O are below 1e-3 of the derivative's scale."""
    for causal, lq, lk in ((True, [40, 9], [40, 9]), (False, [33], [50]), (True, [7], [90])):
        t = make(lq, lk, 4, 2, 32, torch.float32, 11)
        cq, ck = (torch.tensor(ends(x), dtype=torch.int32).cuda() for x in (lq, lk))
        loss = lambda q, k, v: float((F.attention_fwd(q, k, v, cq, ck, causal)[0].double() * t["dO"].double()).sum())
        O, lse = F.attention_fwd(t["q"], t["k"], t["v"], cq, ck, causal)
        grads = dict(zip("qkv", F.attention_bwd(t["dO"], t["q"], t["k"], t["v"], O, lse, cq, ck, causal)))
        arg = {n: t[n] for n in "qkv"}
        for n, g in grads.items():
            d = g / g.norm() + 0.3 * torch.randn_like(g) / g.numel() ** 0.5
            e = 3e-2
            diff = (loss(**{**arg, n: t[n] + e * d}) - loss(**{**arg, n: t[n] - e * d})) / (2 * e)
            assert abs(diff - float((g * d).sum())) <= 3e-3 * float(g.norm() * d.norm()), n


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_repeatable(F, dt):
    lengths = [200, 31, 513]
    t = make(lengths, lengths, 8, 2, 128, DT[dt], 12)
    cu = torch.tensor(ends(lengths), dtype=torch.int32).cuda()
    first = None
    for _ in range(3):
        O, lse = F.attention_fwd(t["q"], t["k"], t["v"], cu)
        now = (O, lse, *F.attention_bwd(t["dO"], t["q"], t["k"], t["v"], O, lse, cu))
        first = first or now
        assert all(torch.equal(a, b) for a, b in zip(first, now))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_graph_replays(F, dt):
    lengths = [90, 40]
    t = make(lengths, lengths, 4, 2, 128, DT[dt], 13)
    cu = torch.tensor(ends(lengths), dtype=torch.int32).cuda()
    ws = F.workspace(F.attention_workspace_size(t["q"], t["k"], 2))
    O, lse = torch.empty_like(t["q"]), torch.empty(4, 130).cuda()
    out = tuple(torch.empty_like(t[n]) for n in "qkv")

    def step():
        F.attention_fwd(t["q"], t["k"], t["v"], cu, ws=ws, out=O, lse=lse)
        F.attention_bwd(t["dO"], t["q"], t["k"], t["v"], O, lse, cu, ws=ws, out=out)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(3):
        new = make(lengths, lengths, 4, 2, 128, DT[dt], 20 + i)
        for n in t:
            t[n].copy_(new[n])
        step()
        torch.cuda.synchronize()
        eager = [x.clone() for x in (O, lse, *out)]
        for x in (O, lse, *out):
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, (O, lse, *out)))


def test_bad_ends_raise_the_domain_flag(F):
    t = make([64], [64], 2, 2, 64, torch.bfloat16, 14)
    for cu in ([0, 40, 20, 64], [0, 30, 65], [-1, 30, 64], [0, 30, 2 ** 31 - 1]):
        ws = F.workspace(F.attention_workspace_size(t["q"], t["k"], 8))
        c = torch.tensor(cu, dtype=torch.int32).cuda()
        O, lse = F.attention_fwd(t["q"], t["k"], t["v"], c, ws=ws, out=torch.zeros_like(t["q"]),
                                 lse=torch.zeros(2, 64).cuda())
        assert F.check_flags(ws) == F.ERR_DOMAIN
        F.attention_bwd(t["dO"], t["q"], t["k"], t["v"], O, lse, c, ws=ws)
        assert F.check_flags(ws) == F.ERR_DOMAIN
        assert F.check_flags(ws) == F.OK


def test_no_tokens(F):
    e = torch.empty(0, 4, 64).cuda()
    O, lse = F.attention_fwd(e, e, e, torch.zeros(1, dtype=torch.int32).cuda())
    assert O.shape == (0, 4, 64) and lse.shape == (4, 0)
    q = torch.randn(3, 4, 64).cuda()
    O, lse = F.attention_fwd(q, e, e, causal=False)
    assert torch.equal(O, torch.zeros_like(q)) and torch.isneginf(lse).all()
    dq, dk, dv = F.attention_bwd(q, q, e, e, O, lse, causal=False)
    assert torch.equal(dq, torch.zeros_like(q)) and dk.shape == (0, 4, 64)
    k = torch.randn(5, 4, 64).cuda()
    O, lse = F.attention_fwd(e, k, k, causal=False)
    dq, dk, dv = F.attention_bwd(e, e, k, k, O, lse, causal=False)
    assert torch.equal(dk, torch.zeros_like(k)) and torch.equal(dv, torch.zeros_like(k))


def test_refusals(F):
    q, k = torch.randn(8, 4, 64).cuda(), torch.randn(8, 2, 64).cuda()
    for call, status in ((lambda: F.attention_fwd(torch.randn(8, 3, 64).cuda(), k, k), F.ERR_SHAPE),
                         (lambda: F.attention_fwd(torch.randn(8, 4, 136).cuda(), torch.randn(8, 4, 136).cuda(),
                                                  torch.randn(8, 4, 136).cuda()), F.ERR_SHAPE),
                         (lambda: F.attention_fwd(*(torch.randn(8, 4, 20).cuda() for _ in range(3))), F.ERR_SHAPE),
                         (lambda: F.attention_fwd(q, k, k, scale=float("inf")), F.ERR_CONFIG),
                         (lambda: F.attention_fwd(torch.randn(8, 4 * 64 + 1).cuda()[:, :256].unflatten(1, (4, 64)), k, k),
                          F.ERR_SHAPE)):
        with pytest.raises(F.FocusError) as e:
            call()
        assert e.value.status == status
    with pytest.raises(TypeError):
        F.attention_fwd(q.half(), k.half(), k.half())
    with pytest.raises(ValueError):
        F.attention_fwd(q, k, k.bfloat16())
    with pytest.raises(ValueError):
        F.attention_fwd(q, k, k[:4])
    with pytest.raises(ValueError):
        F.attention_fwd(q, k, k, torch.zeros(3, dtype=torch.int64).cuda())
    with pytest.raises(ValueError):
        F.attention_fwd(q.transpose(0, 1), k, k)
    with pytest.raises(ValueError):
        F.attention_fwd(q, k, k, lse=torch.empty(8, 4).cuda())


def test_refuses_what_would_reach_a_kernel_wrongly(F):
    """Tensors of the host, and tokens that share their memory (a broadcast tensor)."""
    q = torch.zeros(4, 2, 64, dtype=torch.bfloat16, device="cuda")
    cu = torch.tensor([0, 4], dtype=torch.int32)
    wide = q[:1].expand(4, 2, 64)
    O, lse = F.attention_fwd(q, q, q)
    for call in (lambda: F.attention_fwd(q, q.cpu(), q), lambda: F.attention_fwd(q, q, q, cu),
                 lambda: F.attention_fwd(q.cpu(), q, q), lambda: F.attention_fwd(q, wide, wide),
                 lambda: F.attention_bwd(q, q, q, q, O, lse.cpu()), lambda: F.attention_bwd(q, wide, q, q, O, lse),
                 lambda: F.attention_bwd(q, q, q, q, O, lse, out=(q, wide, q))):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("n", [9, 64, 75, 140])
def test_many_sequences_of_different_lengths(F, n, dt):
    """Every tile is taken once, whatever the lengths of the sequences whose tiles are given out together."""
    g = torch.Generator().manual_seed(n)
    lk = [int(x) for x in torch.randint(0, 60, (n,), generator=g)]
    for i in range(0, n, 13):
        lk[i] = 200 + 5 * i
    lq = [x if i % 3 else x // 2 for i, x in enumerate(lk)]
    run_case(F, lk, lk, 2, 1, 32, dt, True, seed=n)
    run_case(F, lq, lk, 4, 2, 16, dt, True, seed=n + 1)
