"""GPU tests of focus_clip_grad_norm against the definition in float64.

Bounds. Squares of fp32 and bf16 numbers are exact in fp64 and their sum of n terms is off by n 2^-53 of itself at most, the root by
half of that: 1e-9 for up to 2^24 elements. A scaled gradient is one fp32 factor (off by 2^-24) times an fp32 number, rounded
once to the tensor's type: 2^-23 of the value, in bf16 2^-8 and 2^-23.
"""
import math

import pytest
import torch

from gpu_common import announce, require_gpu

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def F():
    return require_gpu()


def make(sizes, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [(torch.randn(n, generator=g, device="cuda") * scale * 10.0 ** -(i % 4)).to(dt) for i, (n, dt) in enumerate(sizes)]


def norm_of(grads):
    return math.sqrt(sum(float(g.double().square().sum()) for g in grads))


def check(F, grads, max_norm, out=None, before=None):
    before = before or [g.clone() for g in grads]
    want = norm_of(before)
    ws = F.workspace(F.clip_grad_norm_workspace_size(len(grads)))
    norm = F.clip_grad_norm(grads, max_norm, out=out, ws=ws)
    assert norm.dtype == torch.float64 and abs(norm.item() - want) <= 1e-9 * want
    factor = max_norm / want if want > max_norm else 1.0
    for g, b, o in zip(grads, before, grads if out is None else out):
        if o is None:
            continue
        ref = b.double() * factor
        if factor == 1.0:
            assert torch.equal(o, b)
        else:
            lim = (2.0 ** -23 + (2.0 ** -8 if b.dtype == BF else 0.0)) * ref.abs() + 2.0 ** -149
            assert ((o.double() - ref).abs() <= lim).all()
        if o is not g:
            assert torch.equal(g, b)
    assert F.check_flags(ws) == F.OK
    return norm


SETS = {"one": [(1, F32)], "odd": [(7, F32), (8191, BF), (8193, F32), (1, BF), (0, F32), (13, BF)],
        "layer": [(256 * 8, F32), (256 * 32, F32)], "group": [(100 + 13 * i, (F32, BF)[i % 2]) for i in range(112)],
        "groups": [(50 + 7 * i, (BF, BF, F32)[i % 3]) for i in range(400)], "large": [(20_000_001, F32), (3, BF), (30_000_007, BF)],
        "empty": [(0, F32), (0, BF)], "none": []}


@pytest.mark.parametrize("name", SETS)
@pytest.mark.parametrize("clips", [True, False])
def test_against_definition(F, name, clips):
    announce(f"clip {name} clips={clips}")
    grads = make(SETS[name], 3)
    n = norm_of(grads)
    max_norm = max(n, 1.0) * (0.37 if clips else 1.5)
    before = [g.clone() for g in grads]
    out = [torch.full_like(g, 7.0) for g in grads]
    check(F, grads, max_norm, out=out, before=before)
    check(F, grads, max_norm, before=before)  # in place, afterwards
    assert all(torch.equal(a, b) for a, b in zip(grads, out))


@pytest.mark.parametrize("scale", [1e-30, 1e30])
def test_sizes_whose_squares_fp32_does_not_hold(F, scale):
    announce(f"clip scale {scale}")
    check(F, make([(5000, F32), (4097, BF)], 4, scale), 0.5 * scale)


def test_factors_smaller_than_the_normal_numbers(F):
    grads = make([(1000, F32), (5000, BF)], 5, 1e36)
    check(F, grads, 1e-4)
    check(F, make([(1000, F32), (5000, BF)], 5, 1e36), 1e-4, out=[torch.empty_like(g) for g in grads])


def test_counted_only(F):
    announce("clip counted only")
    grads = make([(1000, F32), (1000, BF), (1000, F32)], 5)
    check(F, grads, 1.0, out=[None, torch.empty_like(grads[1]), grads[2]])
    check(F, grads, 1.0, out=[None] * 3)
    check(F, grads, math.inf)


def test_a_norm_that_is_not_finite(F):
    for value in (math.inf, math.nan):
        announce(f"clip {value}")
        grads = make([(1000, F32), (77, BF)], 6)
        grads[1][5] = value
        before = [g.clone() for g in grads]
        ws = F.workspace(F.clip_grad_norm_workspace_size(2))
        norm = F.clip_grad_norm(grads, 1.0, ws=ws)
        assert not math.isfinite(norm.item())
        assert F.check_flags(ws) == F.ERR_DOMAIN and F.check_flags(ws) == F.OK
        assert torch.equal(grads[0], before[0])


def test_a_plan_is_called_again(F):
    announce("clip plan")
    grads = make([(3000, F32), (500, BF)], 7)
    plan = F.GradTensors(grads, [torch.empty_like(g) for g in grads])
    ws = F.workspace(F.clip_grad_norm_workspace_size(2))
    for k in range(3):
        for g in grads:
            g.mul_(1.5)
        want = norm_of(grads)
        assert abs(F.clip_grad_norm(plan, 0.1, ws=ws).item() - want) <= 1e-9 * want
        assert abs(norm_of(plan.out) - 0.1) <= 2e-3


def test_captured(F):
    announce("clip captured")
    grads = make([(3000, F32), (70000, BF)] + [(10, F32)] * 130, 8)
    out = [torch.empty_like(g) for g in grads]
    plan, ws = F.GradTensors(grads, out), F.workspace(F.clip_grad_norm_workspace_size(len(grads)))
    norm = torch.empty(1, dtype=torch.float64, device="cuda")
    F.clip_grad_norm(plan, 0.5, ws=ws, norm=norm)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        F.clip_grad_norm(plan, 0.5, ws=ws, norm=norm)
    for k in range(3):
        for g in grads:
            g.mul_(0.7)
        graph.replay()
        got = [norm.clone()] + [o.clone() for o in out]
        F.clip_grad_norm(plan, 0.5, ws=ws, norm=norm)
        assert all(torch.equal(a, b) for a, b in zip(got, [norm] + out)), k


def test_refusals(F):
    a, flat = torch.ones(64, device="cuda"), torch.ones(256, device="cuda")
    with pytest.raises(ValueError):
        F.clip_grad_norm([a], 1.0, out=[a[:32]])
    with pytest.raises(ValueError):
        F.clip_grad_norm([a], 1.0, out=[a, a])
    with pytest.raises(ValueError):
        F.clip_grad_norm([torch.ones(64)], 1.0)
    with pytest.raises(TypeError):
        F.clip_grad_norm([a.half()], 1.0)
    with pytest.raises(ValueError):
        F.clip_grad_norm([a], 1.0, norm=torch.empty(1, device="cuda"))
    for grads, out in (([a, a], None), ([a, a], [a, None]), ([flat[:64]], [flat[32:96]]), ([a, flat[:64]], [flat[4:68], None]),
                       ([flat[:64], flat[64:128]], [flat[128:192], flat[160:224]])):
        with pytest.raises(F.FocusError) as e:
            F.clip_grad_norm(grads, 1.0, out=out)
        assert e.value.status == F.ERR_SHAPE
    for bad in (0.0, -1.0, math.nan):
        with pytest.raises(F.FocusError) as e:
            F.clip_grad_norm([a], bad)
        assert e.value.status == F.ERR_CONFIG
    assert F.clip_grad_norm([a, a], 1.0, out=[None, None]).item() == pytest.approx(math.sqrt(128))
