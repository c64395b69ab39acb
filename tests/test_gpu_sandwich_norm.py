"""GPU tests of focus_sandwich_norm_fwd / focus_sandwich_norm_bwd against the definition in float64.

Bounds. All arithmetic is fp32. A sum over C terms is off by less than (C / 64 + 16) 2^-24 of the sum of magnitudes, 2e-5 with
C <= 17,000; the results depend on the statistics of two norms and, backward, on two more means per norm, each of which
scales a result of the row's size once: fp32 results are held to 6e-5 of max(|value|, rms of the row), bf16 results to that
plus half a step, 2^-8 of the value. A sum over tokens is held to 6e-5 (what each term may be off) + 1e-5 (its own
additions: at most 64 rows in fp32 per workgroup, then fp64) of the sum of its terms' magnitudes.
The gradients of a norm's input are differences, rstd (P - mean P - xb mean(P xb)), whose operands may cancel (with one feature
all but eps of them does): each operand is off by the above of its own size, at most 3 rstd rms(P) in a row's root mean square, so
"the row's size" is that of rstd P there. What is computed from the gradient D of Y (dX, dB, dgate, the sums) has D's error, the above
of |dY| + rstd rms(G), as a factor. A normalised feature near 0 is a difference too, (h - mean) rstd: it is off by 2^-24 of h and of the
mean, each up to some times its row's root mean square, 1, so that factors xb and xy (and U's xb) count as 1 where they are smaller.
"""
import pytest
import torch

from gpu_common import announce, require_gpu

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
NAMES = ("w_post", "w_pre", "b_post", "b_pre")


@pytest.fixture(scope="module")
def F():
    return require_gpu()


def make(T, C, dt, seed, gate="feature", bias=False, wdt=None):
    g = torch.Generator().manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g)
    ch = 1.0 + 19.0 * (torch.rand(C, generator=g) < 0.02)
    t = {"X": rnd(T, C) * ch + 0.3, "B": rnd(T, C) * 0.4 - 0.2, "w_post": 1.0 + 0.2 * rnd(C), "w_pre": 1.0 + 0.2 * rnd(C),
         "b_post": 0.1 * rnd(C), "b_pre": 0.1 * rnd(C), "dN": rnd(T, C), "dY": 0.5 * rnd(T, C),
         "gate": {"none": None, "feature": 0.5 + 0.2 * rnd(C), "token": torch.sigmoid(rnd(T, C))}[gate]}
    if not bias:
        t["b_post"] = t["b_pre"] = None
    per_feature = NAMES + (("gate",) if gate == "feature" else ())
    return {k: None if v is None else v.to(wdt or dt if k in per_feature else dt).cuda() for k, v in t.items()}


def params(t):
    return dict(b_post=t["b_post"], b_pre=t["b_pre"], gate=t["gate"])


def reference(t, layer, eps, scale, with_dy=True):
    """Outputs, gradients and the sums of the magnitudes of the token sums' terms, in float64 by autograd on the host."""
    d = {k: None if v is None else v.double().cpu().requires_grad_(True) for k, v in t.items()}

    def norm(h):
        c = h - h.mean(1, keepdim=True) if layer else h
        return c / torch.sqrt((c * c).mean(1, keepdim=True) + eps)

    T = d["X"].shape[0]
    rows = {k: d[k][None].expand(T, -1) for k in NAMES if d[k] is not None}  # a row of its own for every token
    feature = d["gate"] is not None and d["gate"].dim() == 1
    if feature:
        rows["gate"] = d["gate"][None].expand(T, -1)
    gate = rows.get("gate", d["gate"])
    xb = norm(d["B"])
    u = xb * rows["w_post"]
    u = u + rows["b_post"] if "b_post" in rows else u
    y = scale * d["X"] + (u if gate is None else gate * u)
    xy = norm(y)
    n = xy * rows["w_pre"]
    n = n + rows["b_pre"] if "b_pre" in rows else n
    wrt = {"X": d["X"], "B": d["B"], **rows}
    if d["gate"] is not None and not feature:
        wrt["gate"] = d["gate"]
    f = (n * d["dN"].detach()).sum() + ((y * d["dY"].detach()).sum() if with_dy else 0.0)
    grads = dict(zip(wrt, torch.autograd.grad(f, list(wrt.values()))))
    # sizes that the bounds go by
    with torch.no_grad():
        rms = lambda x: x.square().mean(1, keepdim=True).sqrt()
        rstd = lambda h: 1.0 / torch.sqrt(((h - h.mean(1, keepdim=True) if layer else h) ** 2).mean(1, keepdim=True) + eps)
        size_d = rstd(y) * rms(d["dN"] * rows["w_pre"]) + (d["dY"].abs() if with_dy else 0.0)
        of_gate = torch.ones_like(xb) if gate is None else gate.abs()
        sizes = {"X": abs(scale) * size_d, "B": rstd(d["B"]) * rms(size_d * of_gate * rows["w_post"]), "b_post": size_d * of_gate,
                 "gate": size_d * (xb.abs().clamp(min=1.0) * rows["w_post"].abs() + (rows["b_post"].abs() if "b_post" in rows else 0.0)),
                 "w_post": size_d * of_gate * xb.abs().clamp(min=1.0), "w_pre": d["dN"].abs() * xy.abs().clamp(min=1.0),
                 "b_pre": d["dN"].abs()}
    grads = {k: (v, sizes[k]) for k, v in grads.items()}
    return y.detach(), n.detach(), grads, rows


def near(got, ref, what, dt, tol=6e-5):
    got = got.double().cpu()
    ref, size = ref if isinstance(ref, tuple) else (ref, 0.0 * ref)
    size = torch.maximum(size, torch.maximum(ref.abs(), ref.square().mean(1, keepdim=True).sqrt()))
    lim = tol * size + (2.0 ** -8 if dt == "bf16" else 2.0 ** -24) * ref.abs() + 1e-30
    bad = ~((got - ref).abs() <= lim)
    assert not bad.any(), (what, int(bad.sum()), float(((got - ref).abs() / lim).max()))


def near_sum(got, terms, what):
    ref, size = terms[0].sum(0), torch.maximum(terms[0].abs(), terms[1]).sum(0)
    bad = ~((got.double().cpu() - ref).abs() <= 7e-5 * size + 2.0 ** -24 * ref.abs() + 1e-30)
    assert not bad.any(), (what, int(bad.sum()), float(((got.double().cpu() - ref).abs() / size).max()))


def check(F, t, dt, kind, scale, with_dy=True, eps=1e-5):
    k = F.NORM_LAYER if kind == "layer" else F.NORM_RMS
    args = dict(params(t), residual_scale=scale, kind=k, eps=eps)
    Y, N, stats = F.sandwich_norm_fwd(t["X"], t["B"], t["w_post"], t["w_pre"], **args)
    dX, dB, grads = F.sandwich_norm_bwd(t["dN"], t["dY"] if with_dy else None, t["X"], t["B"], t["w_post"], t["w_pre"], stats, **args)
    torch.cuda.synchronize()
    y, n, ref, rows = reference(t, kind == "layer", eps, scale, with_dy)
    near(Y, y, "Y", dt)
    near(N, n, "N", dt)
    near(dX, ref["X"], "dX", dt)
    near(dB, ref["B"], "dB", dt)
    for name in NAMES + ("gate",):
        if name in rows:
            assert grads[name].dtype == torch.float32
            near_sum(grads[name], ref[name], "d" + name)
        elif name in ref:
            near(grads[name], ref[name], "d" + name, dt)
        else:
            assert grads[name] is None
    return Y, N, stats, dX, dB, grads


SHAPES = [(1, 1), (3, 7), (1, 8192), (5, 64), (129, 65), (37, 1001), (66, 2560), (9, 2561), (18, 4096), (7, 8181), (3, 8200),
          (1030, 96), (4101, 40), (2, 16400)]


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("T,C", SHAPES)
def test_against_definition(F, T, C, dt, kind):
    for gate, bias, wdt, with_dy in (("feature", False, None, True), ("token", True, torch.float32, True), ("none", False, None, False)):
        announce(f"sandwich {kind} {dt} T={T} C={C} gate={gate} bias={bias}")
        if kind == "layer" and C == 1:
            continue  # a layer norm of one feature is its shift
        check(F, make(T, C, DT[dt], T * 31 + C, gate, bias, wdt), dt, kind, 0.8, with_dy)


@pytest.mark.parametrize("which", ["b_post", "b_pre"])
@pytest.mark.parametrize("gate", ["none", "feature", "token"])
def test_one_shift_alone(F, gate, which):
    announce(f"sandwich {which} alone, gate {gate}")
    t = make(21, 328, torch.float32, 5, gate, True)
    t["b_pre" if which == "b_post" else "b_post"] = None
    check(F, t, "f32", "rms", 1.0)


def test_means_that_dwarf_the_differences(F):
    # a branch output whose mean is 300 times its spread: the variance is of differences from the mean
    announce("sandwich large means")
    t = make(9, 1500, torch.float32, 6, "feature", True)
    t["B"] += 120.0
    k = F.NORM_LAYER
    Y, N, _ = F.sandwich_norm_fwd(t["X"], t["B"], t["w_post"], t["w_pre"], **params(t), kind=k)
    y, n, _, _ = reference(t, True, 1e-5, 1.0)
    # B - mean is off by the mean's rounding and its own: 2 x 120 x 2^-24 of a spread of 0.4, 4e-5, twice in a result
    near(Y, y, "Y", "f32", 2e-4)
    near(N, n, "N", "f32", 2e-4)


def test_rows_of_zeros(F):
    # rstd is 1 / sqrt(eps): outputs are the shifts, gradients finite
    announce("sandwich zeros")
    t = make(4, 96, torch.bfloat16, 7, "feature", True)
    t["X"].zero_(), t["B"].zero_()
    Y, N, _, dX, dB, _ = check(F, t, "bf16", "rms", 1.0)
    assert torch.isfinite(dX.float()).all() and torch.isfinite(dB.float()).all()


@pytest.mark.parametrize("C", [96, 2560, 8200])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_outputs_over_inputs(F, C, dt):
    announce(f"sandwich in place {dt} C={C}")
    t = make(11, C, DT[dt], 8, "token", False)
    ws = F.workspace(F.sandwich_norm_workspace_size(11, C))
    args = dict(residual_scale=0.7, kind=F.NORM_RMS, ws=ws)
    Y, N, stats = F.sandwich_norm_fwd(t["X"], t["B"], t["w_post"], t["w_pre"], gate=t["gate"], **args)
    dX, dB, g = F.sandwich_norm_bwd(t["dN"], t["dY"], t["X"], t["B"], t["w_post"], t["w_pre"], stats, gate=t["gate"], **args)
    for place in ("X", "B", "gate"):
        c = {k: v.clone() if v is not None else None for k, v in t.items()}
        other = {"X": "B", "B": "gate", "gate": "X"}[place]
        Y2, N2, _ = F.sandwich_norm_fwd(c["X"], c["B"], c["w_post"], c["w_pre"], gate=c["gate"], out=c[place], n_out=c[other], **args)
        assert torch.equal(Y2, Y) and torch.equal(N2, N), place
    for places in (("dN", "dY", "gate"), ("X", "B", "dN"), ("dY", "gate", "X"), ("gate", "X", "B"), ("B", "dN", "dY")):
        c = {k: v.clone() if v is not None else None for k, v in t.items()}
        dX2, dB2, g2 = F.sandwich_norm_bwd(c["dN"], c["dY"], c["X"], c["B"], c["w_post"], c["w_pre"], stats, gate=c["gate"],
                                           out=c[places[0]], b_out=c[places[1]], gate_out=c[places[2]], **args)
        assert torch.equal(dX2, dX) and torch.equal(dB2, dB), places
        assert all(torch.equal(g2[n], g[n]) for n in ("w_post", "w_pre", "gate")), places
    assert F.check_flags(ws) == F.OK


def test_gradients_against_differences(F):
    announce("sandwich differences")
    t = make(6, 72, torch.float32, 9, "feature", True)
    args = dict(params(t), residual_scale=0.9, kind=F.NORM_LAYER)
    _, _, stats = F.sandwich_norm_fwd(t["X"], t["B"], t["w_post"], t["w_pre"], **args)
    dX, dB, grads = F.sandwich_norm_bwd(t["dN"], t["dY"], t["X"], t["B"], t["w_post"], t["w_pre"], stats, **args)
    got = {"X": dX, "B": dB, **grads}
    g = torch.Generator().manual_seed(3)
    for name in ("X", "B", "w_post", "w_pre", "b_post", "b_pre", "gate"):
        step = torch.randn(t[name].shape, generator=g, dtype=torch.float64)
        values = []
        for sign in (1.0, -1.0):
            c = {k: v.double().cpu() if v is not None else None for k, v in t.items()}
            c[name] = c[name] + sign * 1e-5 * step
            y, n, _, _ = reference(c, True, 1e-5, 0.9)
            values.append(float(((n * c["dN"]).sum() + (y * c["dY"]).sum()).detach()))
        want = (values[0] - values[1]) / 2e-5
        have = (got[name].double().cpu() * step)
        # the difference's own error is (1e-5)^2 of the third derivative, the kernel's 6e-5 of each term
        assert abs(float(have.sum()) - want) <= 1e-4 * float(have.abs().sum()) + 1e-6, name


def test_the_same_bits_twice_and_on_another_stream(F):
    announce("sandwich determinism")
    t = make(1500, 2560, torch.bfloat16, 10, "token", True)
    args = dict(params(t), kind=F.NORM_LAYER)

    def go():
        Y, N, stats = F.sandwich_norm_fwd(t["X"], t["B"], t["w_post"], t["w_pre"], **args)
        dX, dB, g = F.sandwich_norm_bwd(t["dN"], t["dY"], t["X"], t["B"], t["w_post"], t["w_pre"], stats, **args)
        return [Y, N, stats, dX, dB] + [g[n] for n in sorted(g)]

    a = go()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b = go()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_nothing_to_do(F):
    for T, C in ((0, 64), (4, 0), (0, 0)):
        t = make(T, C, torch.float32, 1, "feature", True)
        Y, N, stats = F.sandwich_norm_fwd(t["X"], t["B"], t["w_post"], t["w_pre"], **params(t))
        dX, dB, g = F.sandwich_norm_bwd(t["dN"], t["dY"], t["X"], t["B"], t["w_post"], t["w_pre"], stats, **params(t))
        assert Y.shape == dX.shape == (T, C) and all(v.shape == (C,) and not v.any() for v in g.values())


def test_refusals(F):
    t = make(4, 64, torch.float32, 1, "token")
    other = torch.empty(4, 64, device="cuda", dtype=torch.bfloat16)
    call = lambda **kw: F.sandwich_norm_fwd(**{**dict(X=t["X"], B=t["B"], w_post=t["w_post"], w_pre=t["w_pre"], gate=t["gate"]), **kw})
    for kw in (dict(B=other), dict(w_pre=t["w_pre"][:32]), dict(w_pre=t["w_pre"].bfloat16()), dict(gate=t["gate"][:3]),
               dict(gate=other), dict(out=other), dict(b_post=torch.empty(64))):
        with pytest.raises((ValueError, TypeError)):
            call(**kw)
    flat = torch.empty(8, 64, device="cuda")
    for kw in (dict(out=flat[:4], n_out=flat[:4]), dict(X=flat[:4], out=flat[2:6]), dict(out=flat[:4], n_out=flat[1:5])):
        with pytest.raises(F.FocusError) as e:
            call(**kw)
        assert e.value.status == F.ERR_SHAPE
