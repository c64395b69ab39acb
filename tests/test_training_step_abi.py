"""Host-side checks of the sandwich norm, linear cross entropy and gradient clipping entry points (no kernel is launched).

Every call carries an argument that a check must refuse, or sizes of nothing; pointers are never dereferenced.
"""
import ctypes
import math

import pytest

from paper_2608_01847_amd import focus

at = lambda i: ctypes.c_void_p((1 << 30) + (i << 24))  # tensors 16 MB apart
BIG = 1 << 34


@pytest.fixture(scope="module")
def L():
    if not focus.LIBRARY.exists():
        pytest.skip("libfocus.so is not built")
    return focus.lib()


@pytest.fixture()
def cpu_only():
    import torch
    if torch.cuda.is_available():
        pytest.skip("argument-check tests run in the CPU suite only")


def fwd(L, kind=1, gk=0, eps=1e-5, scale=1.0, X=at(0), B=at(1), dt=1, T=4, C=64, w1=at(2), b1=None, gate=None, w2=at(3), b2=None,
        wdt=1, Y=at(4), N=at(5), stats=at(6), ws=at(9), size=BIG, cfg=True):
    c = ctypes.byref(focus.SandwichConfig(kind, gk, eps, scale)) if cfg else None
    return L.focus_sandwich_norm_fwd(c, X, B, dt, T, C, w1, b1, gate, w2, b2, wdt, Y, N, stats, ws, size, None)


def bwd(L, kind=1, gk=0, eps=1e-5, scale=1.0, dN=at(10), dY=None, X=at(0), B=at(1), dt=1, T=4, C=64, w1=at(2), b1=None, gate=None,
        w2=at(3), wdt=1, stats=at(6), dX=at(11), dB=at(12), dg=None, dw1=at(13), db1=None, dw2=at(14), db2=None, ws=at(9), size=BIG,
        cfg=True):
    c = ctypes.byref(focus.SandwichConfig(kind, gk, eps, scale)) if cfg else None
    return L.focus_sandwich_norm_bwd(c, dN, dY, X, B, dt, T, C, w1, b1, gate, w2, wdt, stats, dX, dB, dg, dw1, db1, dw2, db2, ws,
                                     size, None)


def test_sandwich_checks(L, cpu_only):
    F = focus
    off = ctypes.c_void_p(at(0).value + 8)
    inside = ctypes.c_void_p(at(0).value + 64)
    common = ((F.ERR_NULL, {"cfg": False}), (F.ERR_CONFIG, {"kind": 2}), (F.ERR_CONFIG, {"gk": 3}), (F.ERR_CONFIG, {"gk": -1}),
              (F.ERR_CONFIG, {"eps": -1.0}), (F.ERR_CONFIG, {"eps": math.nan}), (F.ERR_CONFIG, {"scale": math.inf}),
              (F.ERR_CONFIG, {"gate": at(7)}), (F.ERR_NULL, {"gk": 1}), (F.ERR_NULL, {"gk": 2}), (F.ERR_DTYPE, {"dt": 2}),
              (F.ERR_DTYPE, {"wdt": -1}), (F.ERR_SHAPE, {"T": -1}), (F.ERR_SHAPE, {"T": 1 << 31}), (F.ERR_SHAPE, {"C": (1 << 24) + 1}),
              (F.ERR_SHAPE, {"T": 1 << 30, "C": 1 << 20}), (F.ERR_NULL, {"X": None}), (F.ERR_NULL, {"B": None}),
              (F.ERR_NULL, {"w1": None}), (F.ERR_NULL, {"w2": None}), (F.ERR_SHAPE, {"X": off}), (F.ERR_WORKSPACE, {"ws": None}),
              (F.ERR_WORKSPACE, {"size": 255}), (F.OK, {"C": 0}))
    for status, kw in common:
        assert fwd(L, **kw) == status, kw
        assert bwd(L, **kw) == status, kw
    for status, kw in ((F.ERR_NULL, {"Y": None}), (F.ERR_NULL, {"N": None}), (F.OK, {"T": 0, "X": None}), (F.ERR_SHAPE, {"N": at(4)}),
                       (F.ERR_SHAPE, {"Y": inside}), (F.ERR_SHAPE, {"Y": at(2)}), (F.ERR_SHAPE, {"stats": at(1)}),
                       (F.ERR_SHAPE, {"N": at(6)})):
        assert fwd(L, **kw) == status, kw
    need = F.sandwich_norm_workspace_size(1000, 64)
    for status, kw in ((F.ERR_NULL, {"dN": None}), (F.ERR_NULL, {"stats": None}), (F.ERR_NULL, {"dX": None}), (F.ERR_NULL, {"dB": None}),
                       (F.ERR_NULL, {"dw1": None}), (F.ERR_NULL, {"dw2": None}), (F.ERR_CONFIG, {"dg": at(15)}),
                       (F.ERR_SHAPE, {"dB": at(11)}), (F.ERR_SHAPE, {"dX": inside}), (F.ERR_SHAPE, {"dw1": at(14)}),
                       (F.ERR_SHAPE, {"dw1": at(0)}), (F.ERR_SHAPE, {"dX": at(6)}), (F.ERR_SHAPE, {"db2": at(3)}),
                       (F.ERR_WORKSPACE, {"T": 1000, "size": need - 1})):
        assert bwd(L, **kw) == status, kw


def ce_fwd(L, X=at(0), W=at(1), dt=1, T=4, V=100, K=64, t=at(2), logp=at(3), lse=at(4), ws=at(9), size=BIG):
    return L.focus_linear_ce_fwd(X, W, dt, T, V, K, t, logp, lse, ws, size, None)


def ce_bwd(L, X=at(0), W=at(1), dt=1, T=4, V=100, K=64, t=at(2), lse=at(4), g=at(5), h=None, dX=at(6), dW=at(7), wdt=1, ws=at(9),
           size=BIG):
    return L.focus_linear_ce_bwd(X, W, dt, T, V, K, t, lse, g, h, dX, dW, wdt, ws, size, None)


def test_linear_ce_checks(L, cpu_only):
    F = focus
    odd, off = ctypes.c_void_p(at(8).value + 2), ctypes.c_void_p(at(8).value + 8)
    for call in (ce_fwd, ce_bwd):
        for status, kw in ((F.ERR_DTYPE, {"dt": 2}), (F.ERR_SHAPE, {"T": -1}), (F.ERR_SHAPE, {"T": (1 << 24) + 1}), (F.ERR_SHAPE, {"V": 0}),
                           (F.ERR_SHAPE, {"V": (1 << 24) + 1}), (F.ERR_SHAPE, {"K": 0}), (F.ERR_SHAPE, {"K": (1 << 20) + 1}),
                           (F.ERR_NULL, {"X": None}), (F.ERR_NULL, {"W": None}), (F.ERR_NULL, {"lse": None}), (F.ERR_NULL, {"t": None}),
                           (F.ERR_SHAPE, {"X": off}), (F.ERR_SHAPE, {"W": off}), (F.ERR_SHAPE, {"lse": odd}),
                           (F.ERR_SHAPE, {"t": ctypes.c_void_p(at(2).value + 4)}), (F.ERR_WORKSPACE, {"ws": None}),
                           (F.ERR_WORKSPACE, {"size": 256})):
            assert call(L, **kw) == status, (call, kw)
    assert ce_fwd(L, T=0, X=None, lse=None) == F.OK
    assert ce_fwd(L, dt=0, T=(1 << 23) + 1) == F.ERR_SHAPE and ce_bwd(L, dt=0, wdt=0, T=(1 << 23) + 1) == F.ERR_SHAPE
    for kw in ({"lse": at(3)}, {"lse": at(0)}, {"lse": at(1)}, {"logp": at(2)}, {"logp": ctypes.c_void_p(at(4).value + 8)}):
        assert ce_fwd(L, **kw) == F.ERR_SHAPE, kw
    for status, kw in ((F.ERR_NULL, {"g": None}), (F.ERR_NULL, {"dX": None, "dW": None}), (F.ERR_DTYPE, {"wdt": 7}),
                       (F.ERR_DTYPE, {"dt": 0, "wdt": 1}), (F.ERR_SHAPE, {"dX": at(0)}), (F.ERR_SHAPE, {"dW": at(1)}),
                       (F.ERR_SHAPE, {"dW": at(6)}), (F.ERR_SHAPE, {"dX": ctypes.c_void_p(at(4).value)}), (F.OK, {"T": 0, "dW": None})):
        assert ce_bwd(L, **kw) == status, kw


def test_workspace_sizes(L):
    F = focus
    assert F.sandwich_norm_workspace_size(1 << 20, 2560) == 256 + 1024 * 2560 * 16
    sizes = [F.sandwich_norm_workspace_size(T, 64) for T in (0, 1, 3, 4, 5, 100, 5000, 1 << 20)]
    assert sizes == sorted(sizes)
    assert F.sandwich_norm_workspace_size(-1, 64) == 0 and F.sandwich_norm_workspace_size(1 << 30, 1 << 20) == 0
    for backward in (False, True):
        for V, K in ((1, 1), (5003, 1008), (151936, 2560), (1 << 24, 64)):
            sizes = [F.linear_ce_workspace_size(T, V, K, backward) for T in (0, 1, 2, 31, 32, 33, 255, 257, 4096, 8192, 100000, 1 << 20, 1 << 24)]
            assert sizes == sorted(sizes) and sizes[0] >= 256, (V, K, sizes)
    for bad in ((-1, 5, 5), ((1 << 24) + 1, 5, 5), (5, 0, 5), (5, (1 << 24) + 1, 5), (5, 5, 0), (5, 5, (1 << 20) + 1)):
        assert F.linear_ce_workspace_size(*bad) == 0
    assert F.clip_grad_norm_workspace_size(0) >= 256 and F.clip_grad_norm_workspace_size(-1) == 0
    assert F.clip_grad_norm_workspace_size((1 << 20) + 1) == 0


def clip(L, tensors, max_norm=1.0, norm=at(8), ws=at(9), size=BIG, n=None):
    arr = (focus.GradTensor * max(1, len(tensors)))()
    for i, t in enumerate(tensors):
        g, o, count, dt, reserved = t
        arr[i] = focus.GradTensor(g.value if g else None, o.value if o else None, count, dt, reserved)
    return L.focus_clip_grad_norm(arr, len(tensors) if n is None else n, max_norm, norm, ws, size, None)


def test_clip_checks(L, cpu_only):
    F = focus
    ok = (at(0), at(0), 100, 0, 0)
    within = lambda i, bytes_: ctypes.c_void_p(at(i).value + bytes_)
    for status, args, kw in ((F.ERR_CONFIG, [ok], {"max_norm": 0.0}), (F.ERR_CONFIG, [ok], {"max_norm": math.nan}),
                             (F.ERR_SHAPE, [ok], {"n": -1}), (F.ERR_SHAPE, [ok], {"n": (1 << 20) + 1}), (F.ERR_NULL, [ok], {"norm": None}),
                             (F.ERR_SHAPE, [ok], {"norm": within(8, 4)}), (F.ERR_DTYPE, [(at(0), None, 5, 2, 0)], {}),
                             (F.ERR_CONFIG, [(at(0), None, 5, 0, 1)], {}), (F.ERR_SHAPE, [(at(0), None, -1, 0, 0)], {}),
                             (F.ERR_SHAPE, [(at(0), None, (1 << 36) + 1, 0, 0)], {}), (F.ERR_NULL, [(None, None, 5, 0, 0)], {}),
                             (F.ERR_SHAPE, [(within(0, 8), None, 5, 0, 0)], {}), (F.ERR_SHAPE, [(at(0), within(1, 4), 5, 0, 0)], {}),
                             # the same gradient scaled twice, outputs over one another, over another's gradient, over a part of their own
                             (F.ERR_SHAPE, [ok, ok], {}), (F.ERR_SHAPE, [(at(0), at(2), 100, 0, 0), (at(1), within(2, 384), 100, 0, 0)], {}),
                             (F.ERR_SHAPE, [(at(0), within(1, 16), 100, 0, 0), (at(1), None, 100, 0, 0)], {}),
                             (F.ERR_SHAPE, [(at(1), at(1), 100, 0, 0), (at(0), at(1), 1, 0, 0)], {}),
                             (F.ERR_SHAPE, [(at(8), None, 2, 0, 0)], {}), (F.ERR_SHAPE, [ok], {"norm": within(0, 392)}),
                             (F.ERR_SHAPE, [(at(0), at(8), 1, 1, 0)], {}),
                             (F.ERR_SHAPE, [(at(0), within(0, 16), 100, 0, 0)], {}), (F.ERR_WORKSPACE, [ok], {"ws": None}),
                             (F.ERR_WORKSPACE, [ok], {"size": 512})):
        assert clip(L, args, **kw) == status, (args, kw)
    many = [(at(0) if i == 700 else ctypes.c_void_p(at(20).value + 4096 * ((i * 37) % 2000)),) * 2 + (1000, 0, 0) for i in range(2000)]
    assert clip(L, many, size=512) == F.ERR_WORKSPACE  # nothing overlaps: the next check is reached
    many[1500] = (at(0), at(0), 1000, 1, 0)
    assert clip(L, many, size=512) == F.ERR_SHAPE
