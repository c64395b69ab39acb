"""GPU tests of the sums over tokens in focus_sandwich_norm_bwd where a workgroup takes hundreds and thousands of them.

Every token is the same, so that a sum is T times the term, which the call on one token gives. Bound: rows are added up in fp32 in chunks of
64 (where a wave or a workgroup takes more than 4,096, of the root of their number), the chunks' sums in fp32 too, what is left in fp64:
(64 + n / 64 + 4) 2^-24 of the sum for n rows of a workgroup (or of one of its four waves, up to 1,024 features), and 4 x 2^-24 for the roundings of
the term and of the result. One chain of n additions of the same number rounds the same way as long as the sum keeps its exponent: n 2^-25 and
more, 2e-5 to 1e-4 in these cases.
"""
import pytest
import torch

from gpu_common import announce, require_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def F():
    return require_gpu()


@pytest.fixture(autouse=True)
def memory():
    yield
    torch.cuda.empty_cache()


# tokens, features, tokens of a wave or workgroup
CASES = [(1 << 22, 8, 1024), (1 << 24, 24, 4096), (1 << 20, 1032, 1024), (1 << 19, 1001, 128), (1 << 18, 8192, 1024), (1 << 18, 8200, 1024)]


@pytest.mark.parametrize("T,C,n", CASES)
@pytest.mark.parametrize("kind,gate,bias", [("rms", "feature", False), ("layer", "token", True)])
def test_equal_tokens(F, T, C, n, kind, gate, bias):
    announce(f"sandwich sums {T} x {C} {kind} gate={gate}")
    g = torch.Generator().manual_seed(C)
    rnd = lambda *s: torch.randn(*s, generator=g).to(torch.bfloat16).cuda()
    one = {k: rnd(1, C) for k in ("X", "B", "dN", "dY", "gate")}
    w1, w2 = 1.0 + 0.2 * rnd(C), 1.0 + 0.2 * rnd(C)
    b1, b2 = (rnd(C), rnd(C)) if bias else (None, None)

    def sums(t):
        gates = rnd_gate if gate == "feature" else t["gate"]
        args = dict(b_post=b1, b_pre=b2, gate=gates, kind=F.NORM_LAYER if kind == "layer" else F.NORM_RMS)
        Y, N, stats = F.sandwich_norm_fwd(t["X"], t["B"], w1, w2, **args)
        dX, dB, grads = F.sandwich_norm_bwd(t["dN"], t["dY"], t["X"], t["B"], w1, w2, stats, **args, out=Y, b_out=N)
        return dX, dB, grads

    rnd_gate = 0.5 + 0.2 * rnd(C)
    dX, dB, term = sums(one)
    many = {k: v.expand(T, C).contiguous() for k, v in one.items() if k != "gate" or gate == "token"}
    dX2, dB2, got = sums(many)
    assert torch.equal(dX2[-1], dX[0]) and torch.equal(dB2[T // 2], dB[0])
    lim = (64 + n / 64 + 4 + 4) * 2.0 ** -24
    names = ["w_post", "w_pre"] + (["b_post", "b_pre"] if bias else []) + (["gate"] if gate == "feature" else [])
    for name in names:
        want = T * term[name].double()
        err = (got[name].double() - want).abs()
        assert (err <= lim * want.abs()).all(), (name, float((err / want.abs()).max()), lim)


@pytest.mark.parametrize("T,C", [(300007, 72), (70001, 2600), (40009, 8200)])
@pytest.mark.parametrize("kind,gate,bias", [("rms", "token", False), ("layer", "feature", True)])
def test_tokens_of_their_own(F, T, C, kind, gate, bias):
    # every workgroup (wave) has more than one chunk of tokens, the last ones odd. Bound: that of the tests of ordinary sizes, 7e-5 of the sum
    # of the terms' sizes, a normalised feature near 0 counting as 1
    announce(f"sandwich sums of different tokens {T} x {C} {kind}")
    g = torch.Generator(device="cuda").manual_seed(C)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
    X, B, dN, dY = (rnd(T, C) + m for m in (0.2, -0.1, 0.5, 0.0))
    w1, w2 = 1.0 + 0.2 * rnd(C), 1.0 + 0.2 * rnd(C)
    b1, b2 = (0.1 * rnd(C), 0.1 * rnd(C)) if bias else (None, None)
    gates = torch.sigmoid(rnd(T, C)) if gate == "token" else 0.5 + 0.2 * rnd(C)
    args = dict(b_post=b1, b_pre=b2, gate=gates, kind=F.NORM_LAYER if kind == "layer" else F.NORM_RMS, residual_scale=0.9)
    stats = F.sandwich_norm_fwd(X, B, w1, w2, **args)[2]
    _, _, got = F.sandwich_norm_bwd(dN, dY, X, B, w1, w2, stats, **args)
    want = {k: [torch.zeros(C, dtype=torch.float64, device="cuda") for _ in range(2)] for k in ("w_post", "w_pre", "b_post", "b_pre", "gate")}

    def norm(h):
        c = h - h.mean(1, keepdim=True) if kind == "layer" else h
        rstd = 1.0 / torch.sqrt(c.square().mean(1, keepdim=True) + 1e-5)
        return c * rstd, rstd

    step = (1 << 25) // C
    for r in range(0, T, step):
        e = slice(r, min(T, r + step))
        x, b, n, y = (t[e].double() for t in (X, B, dN, dY))
        gate_of = gates[e].double() if gate == "token" else gates.double()
        xb, _ = norm(b)
        u = xb * w1.double() + (b1.double() if bias else 0.0)
        xy, rstd = norm(0.9 * x + gate_of * u)
        G = n * w2.double()
        D = y + rstd * (G - xy * (G * xy).mean(1, keepdim=True) - (G.mean(1, keepdim=True) if kind == "layer" else 0.0))
        size = y.abs() + rstd * G.square().mean(1, keepdim=True).sqrt()
        size_u = xb.abs().clamp(min=1.0) * w1.double().abs() + (b1.double().abs() if bias else 0.0)
        for k, term, of in (("w_post", D * gate_of * xb, size * gate_of.abs() * xb.abs().clamp(min=1.0)), ("b_post", D * gate_of, size * gate_of.abs()),
                            ("w_pre", n * xy, n.abs() * xy.abs().clamp(min=1.0)), ("b_pre", n, n.abs()), ("gate", D * u, size * size_u)):
            want[k][0] += term.sum(0)
            want[k][1] += torch.maximum(of, term.abs()).sum(0)
    for k in ["w_post", "w_pre"] + (["b_post", "b_pre"] if bias else []) + (["gate"] if gate == "feature" else []):
        err = (got[k].double() - want[k][0]).abs()
        assert (err <= 7e-5 * want[k][1]).all(), (k, float((err / want[k][1]).max()))
