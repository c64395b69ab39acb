"""GPU tests of focus_norm_fwd / focus_norm_bwd against the definition in float64.

Bounds. All arithmetic is fp32 on C terms: a sum over a lane's elements, 6 steps over the wave and at most 4 waves, so
its error is below (C / 64 + 16) 2^-24 of the sum of magnitudes; with C <= 17,000 that is 2e-5, and it enters mean, rstd
and the backward's two means, each of which scales a result of size rms once. fp32 results are held to 3e-5 of
max(|value|, rms of the row or column); bf16 results to that plus half a unit in the last place (2^-9 of the value, 2^-8
with the sum's own rounding on either side). Sums over tokens (dw, db): T terms in fp32 per workgroup, then fp64.
"""
import pytest
import torch

from gpu_common import announce, require_gpu

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def F():
    return require_gpu()


def make(T, C, dt, seed, residual=True, wdt=None):
    g = torch.Generator().manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g)
    ch = 1.0 + 19.0 * (torch.rand(C, generator=g) < 0.02)
    t = {"X": rnd(T, C) * ch + 0.5, "R": rnd(T, C) * 0.5 if residual else None, "w": 1.0 + 0.2 * rnd(C), "b": 0.1 * rnd(C),
         "dY": rnd(T, C), "dR": rnd(T, C) * 0.5 if residual else None}
    return {k: None if v is None else v.to(wdt or dt if k in "wb" else dt).cuda() for k, v in t.items()}


def reference(F, t, kind, eps, bias):
    """(Y, H, dX, dw, db) in float64 on the host."""
    d = {k: None if v is None else v.double().cpu() for k, v in t.items()}
    h = d["X"] if d["R"] is None else (d["X"] + d["R"]).to(t["X"].dtype).double()
    C = h.shape[1]
    mean = h.sum(1, keepdim=True) / C if kind == F.NORM_LAYER else torch.zeros(h.shape[0], 1, dtype=torch.float64)
    c = h - mean
    rstd = 1.0 / ((c * c).sum(1, keepdim=True) / C + eps).sqrt()
    xh = c * rstd
    y = xh * d["w"] + (d["b"] if bias else 0.0)
    g = d["dY"] * d["w"]
    dx = g - xh * (g * xh).sum(1, keepdim=True) / C
    if kind == F.NORM_LAYER:
        dx = dx - g.sum(1, keepdim=True) / C
    dx = dx * rstd
    if d["dR"] is not None:
        dx = dx + d["dR"]
    return y, h, dx, (d["dY"] * xh).sum(0), d["dY"].sum(0)


def near(got, ref, what, dim, tol=3e-5):
    got = got.double().cpu() if got.dtype == torch.float32 else got
    half = 0.0
    if got.dtype == torch.bfloat16:
        got, half = got.double().cpu(), 2.0 ** -8
    size = ref.square().mean(dim, keepdim=True).sqrt() if dim is not None else ref.square().mean().sqrt()
    lim = tol * torch.maximum(ref.abs(), size) + half * ref.abs() + 1e-30
    bad = ~((got - ref).abs() <= lim)
    assert not bad.any(), (what, int(bad.sum()), float(((got - ref).abs() / lim).max()))


SHAPES = [(1, 1), (3, 7), (1, 8192), (5, 64), (129, 65), (37, 1001), (66, 2560), (9, 2561), (18, 4096), (7, 8181), (3, 16384),
          (5, 16392), (1030, 96), (4101, 40)]


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("T,C", SHAPES)
def test_norm_against_definition(F, T, C, dt, kind):
    k = F.NORM_LAYER if kind == "layer" else F.NORM_RMS
    for residual, bias, wdt in ((True, False, None), (False, True, torch.float32)):
        announce(f"norm {kind} {dt} T={T} C={C} residual={residual} bias={bias}")
        t = make(T, C, DT[dt], T * 31 + C, residual, wdt)
        b = t["b"] if bias else None
        Y, H, mean, rstd = F.norm_fwd(t["X"], t["w"], b, t["R"], k, 1e-5)
        dX, dw, db = F.norm_bwd(t["dY"], H if residual else t["X"], t["w"], mean, rstd, t["dR"], k, want_bias=bias)
        torch.cuda.synchronize()
        assert (H is not None) == residual and (mean is not None) == (kind == "layer") and (db is not None) == bias
        y, h, dx, rw, rb = reference(F, t, k, 1e-5, bias)
        if residual:
            assert torch.equal(H.double().cpu(), h)
        near(Y, y, "Y", 1)
        if C > 1:
            near(dX, dx, "dX", 1)
        else:  # one feature: the terms cancel to the residual's gradient; what is left is their rounding
            lim = 1e-4 * (t["dY"].double().cpu() * t["w"].double().cpu() * rstd.double().cpu()[:, None]).abs() + 2.0 ** -8 * dx.abs()
            assert ((dX.double().cpu() - dx).abs() <= lim + 1e-30).all()
        near(dw, rw, "dw", None, 3e-5 * max(1.0, (T / 64) ** 0.5))
        if bias:
            near(db, rb, "db", None, 3e-5 * max(1.0, (T / 64) ** 0.5))


def test_large_mean_keeps_its_digits(F):
    # values near 1,000 with differences of size 1: the variance must come from the differences
    g = torch.Generator().manual_seed(5)
    X = (1000.0 + torch.randn(33, 768, generator=g)).cuda()
    w = torch.ones(768).cuda()
    Y, _, _, _ = F.norm_fwd(X, w, eps=0.0)
    d = X.double().cpu()
    c = d - d.mean(1, keepdim=True)
    ref = c / c.square().mean(1, keepdim=True).sqrt()
    # the mean is rounded to a spacing of 6e-5 (2^-14), once more in its sum
    assert (Y.double().cpu() - ref).abs().max() <= 4 * 2.0 ** -14


def test_constant_and_zero_rows(F):
    X = torch.zeros(4, 100)
    X[1] = 3.0
    X[2] = -7.5
    X = X.cuda()
    w, b = torch.full((100,), 2.0).cuda(), torch.full((100,), 0.25).cuda()
    Y, _, mean, rstd = F.norm_fwd(X, w, b, eps=1e-5)
    assert torch.equal(Y, torch.full_like(Y, 0.25))
    assert torch.equal(mean.cpu(), torch.tensor([0.0, 3.0, -7.5, 0.0]))
    Y, _, _, _ = F.norm_fwd(X, w, None, kind=F.NORM_RMS, eps=1e-5)
    assert torch.equal(Y[0].cpu(), torch.zeros(100)) and torch.isfinite(Y).all()


def test_a_bad_row_stays_its_own(F):
    X = torch.randn(9, 200).cuda()
    X[4, 17] = float("nan")
    X[6, 3] = float("inf")
    w = torch.ones(200).cuda()
    Y, _, mean, rstd = F.norm_fwd(X, w)
    keep = [0, 1, 2, 3, 5, 7, 8]
    assert torch.isfinite(Y[keep]).all() and torch.isnan(Y[4]).all() and not torch.isfinite(Y[6]).all()
    dX, _, _ = F.norm_bwd(torch.randn(9, 200).cuda(), X, w, mean, rstd)
    assert torch.isfinite(dX[keep]).all()


@pytest.mark.parametrize("C", [264, 5000, 20000])
def test_gradient_against_differences(F, C):
    """Central differences of L = sum(Y G) along random directions, in fp32: with a step of 1e-2 the third-order term is
    below 1e-3 of the derivative's scale and the rounding of L below 1e-4 of it."""
    T = 6
    for kind in (F.NORM_LAYER, F.NORM_RMS):
        t = make(T, C, torch.float32, C, residual=False)
        t["X"] = torch.randn(T, C, generator=torch.Generator().manual_seed(C)).cuda()
        G = t["dY"]
        loss = lambda X, w, b: float((F.norm_fwd(X, w, b, None, kind, 1e-5)[0].double() * G.double()).sum())
        Y, _, mean, rstd = F.norm_fwd(t["X"], t["w"], t["b"], None, kind, 1e-5)
        dX, dw, db = F.norm_bwd(G, t["X"], t["w"], mean, rstd, None, kind, want_bias=True)
        for name, x, g in (("X", t["X"], dX), ("w", t["w"], dw), ("b", t["b"], db)):
            # a direction that has the gradient in it, so that the derivative is of the gradient's size
            u = g / g.norm() + 0.3 * torch.randn_like(x) / x.numel() ** 0.5
            e = 1e-2 * x.numel() ** 0.5 / u.norm() * (0.1 if name == "X" else 1.0)
            arg = {"X": t["X"], "w": t["w"], "b": t["b"]}
            hi, lo = loss(**{**arg, name: x + e * u}), loss(**{**arg, name: x - e * u})
            want = float((g.double() * u.double()).sum())
            assert abs((hi - lo) / (2 * e) - want) <= 2e-3 * float(g.norm() * u.norm()), name


def test_outputs_in_place_and_repeatable(F):
    t = make(300, 2560, torch.bfloat16, 3)
    Y, H, mean, rstd = F.norm_fwd(t["X"], t["w"], None, t["R"], F.NORM_RMS)
    dX, dw, _ = F.norm_bwd(t["dY"], H, t["w"], None, rstd, t["dR"], F.NORM_RMS)
    X2, dY2 = t["X"].clone(), t["dY"].clone()
    Y2, H2, _, rstd2 = F.norm_fwd(X2, t["w"], None, t["R"], F.NORM_RMS, h_out=X2)
    dX2, dw2, _ = F.norm_bwd(dY2, H2, t["w"], None, rstd2, t["dR"], F.NORM_RMS, out=dY2)
    for a, b in ((Y, Y2), (H, H2), (rstd, rstd2), (dX, dX2), (dw, dw2)):
        assert torch.equal(a, b)
    assert H2.data_ptr() == X2.data_ptr() and dX2.data_ptr() == dY2.data_ptr()


def test_empty_tensors(F):
    w = torch.ones(64).cuda()
    Y, _, mean, rstd = F.norm_fwd(torch.empty(0, 64).cuda(), w)
    assert Y.shape == (0, 64) and rstd.shape == (0,)
    dX, dw, db = F.norm_bwd(torch.empty(0, 64).cuda(), torch.empty(0, 64).cuda(), w, mean, rstd, want_bias=True,
                            dw_out=torch.full((64,), 7.0).cuda(), db_out=torch.full((64,), 7.0).cuda())
    assert torch.equal(dw.cpu(), torch.zeros(64)) and torch.equal(db.cpu(), torch.zeros(64))


def test_other_stream(F):
    t = make(64, 512, torch.float32, 9, residual=False)
    ref = F.norm_fwd(t["X"], t["w"])[0]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = F.norm_fwd(t["X"], t["w"])[0]
    s.synchronize()
    assert torch.equal(ref, got)


def test_refusals(F):
    X, w = torch.randn(4, 64).cuda(), torch.ones(64).cuda()
    with pytest.raises(ValueError):
        F.norm_fwd(X, torch.ones(63).cuda())
    with pytest.raises(ValueError):
        F.norm_fwd(X, w, residual=X[:, :32])
    with pytest.raises(ValueError):
        F.norm_fwd(X.t(), torch.ones(4).cuda())  # not contiguous
    with pytest.raises(ValueError):
        F.norm_fwd(X, w, h_out=X)
    with pytest.raises(TypeError):
        F.norm_fwd(X.half(), w)
    for call in (lambda: F.norm_fwd(X, w, kind=2), lambda: F.norm_fwd(X, w, eps=-1.0), lambda: F.norm_fwd(X, w, eps=float("nan"))):
        with pytest.raises(F.FocusError) as e:
            call()
        assert e.value.status == F.ERR_CONFIG


def test_more_rows_than_one_launch_holds(F):
    """The rows past 2^24 - 1 against a call of their own."""
    T, C, tail = (1 << 24) + 1000, 16, 1500
    X = torch.randn(T, C, device="cuda", generator=torch.Generator("cuda").manual_seed(3)).bfloat16()
    w = torch.linspace(0.5, 1.5, C, device="cuda")
    Y, H, mean, rstd = F.norm_fwd(X, w, residual=X, kind=F.NORM_LAYER)
    y, h, m, r = F.norm_fwd(X[-tail:].contiguous(), w, residual=X[-tail:].contiguous(), kind=F.NORM_LAYER)
    for all_rows, some in ((Y, y), (H, h), (mean, m), (rstd, r)):
        assert torch.equal(all_rows[-tail:], some)


def test_refuses_tensors_of_the_host(F):
    X, w = torch.zeros(3, 16, device="cuda"), torch.ones(16, device="cuda")
    Y, H, mean, rstd = F.norm_fwd(X, w)
    for call in (lambda: F.norm_fwd(X.cpu(), w), lambda: F.norm_fwd(X, w.cpu()), lambda: F.norm_fwd(X, w, residual=X.cpu()),
                 lambda: F.norm_bwd(X, X, w, mean, rstd.cpu()), lambda: F.norm_bwd(X.cpu(), X, w, mean, rstd)):
        with pytest.raises(ValueError):
            call()
