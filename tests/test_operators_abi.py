"""Host-side checks of the norm, attention and token log-probability entry points (no kernel is launched).

Every call carries an argument that a check must refuse, or sizes of nothing; pointers are never dereferenced.
"""
import ctypes

import pytest

from paper_2608_01847_amd import focus

B = ctypes.c_void_p(1 << 20)
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


def norm_fwd(L, kind=0, eps=1e-5, X=B, R=None, dt=1, T=4, C=64, w=B, b=None, wdt=1, H=None, Y=B, mean=None, rstd=None, ws=B,
             size=BIG):
    return L.focus_norm_fwd(kind, eps, X, R, dt, T, C, w, b, wdt, H, Y, mean, rstd, ws, size, None)


def norm_bwd(L, kind=0, dY=B, H=B, dt=1, T=4, C=64, w=B, wdt=1, mean=B, rstd=B, dH=None, dX=B, dw=B, db=None, ws=B, size=BIG):
    return L.focus_norm_bwd(kind, dY, H, dt, T, C, w, wdt, mean, rstd, dH, dX, dw, db, ws, size, None)


def test_norm_checks(L, cpu_only):
    F = focus
    for status, kw in ((F.ERR_CONFIG, {"kind": 2}), (F.ERR_CONFIG, {"eps": -1.0}), (F.ERR_CONFIG, {"eps": float("inf")}),
                       (F.ERR_CONFIG, {"kind": 1, "mean": B}), (F.ERR_CONFIG, {"H": B}), (F.ERR_DTYPE, {"dt": 2}),
                       (F.ERR_DTYPE, {"wdt": -1}), (F.ERR_SHAPE, {"T": -1}), (F.ERR_SHAPE, {"T": 1 << 31}),
                       (F.ERR_SHAPE, {"C": (1 << 24) + 1}), (F.ERR_NULL, {"X": None}), (F.ERR_NULL, {"w": None}),
                       (F.ERR_NULL, {"Y": None}), (F.ERR_NULL, {"R": B}), (F.ERR_SHAPE, {"X": ctypes.c_void_p((1 << 20) + 8)}),
                       (F.ERR_WORKSPACE, {"ws": None}), (F.ERR_WORKSPACE, {"size": 255}), (F.OK, {"T": 0, "X": None}),
                       (F.OK, {"C": 0})):
        assert norm_fwd(L, **kw) == status, kw
    need = F.norm_workspace_size(1000, 64)
    for status, kw in ((F.ERR_CONFIG, {"kind": -1}), (F.ERR_CONFIG, {"kind": 1}), (F.ERR_NULL, {"mean": None}),
                       (F.ERR_NULL, {"rstd": None}), (F.ERR_NULL, {"dw": None}), (F.ERR_NULL, {"dX": None}),
                       (F.ERR_DTYPE, {"dt": 5}), (F.ERR_SHAPE, {"C": -1}), (F.ERR_WORKSPACE, {"T": 1000, "size": need - 1}),
                       (F.OK, {"C": 0, "dw": None})):
        assert norm_bwd(L, **kw) == status, kw


def attn(L, which="fwd", Hq=4, Hkv=2, D=64, causal=1, scale=0.125, reserved=0, strides=(0,) * 6, q=B, k=B, v=B, dt=1, Tq=8,
         Tk=8, cu_q=None, cu_k=None, n=1, O=B, lse=B, ws=B, size=BIG, cfg=True, dO=B, dq=B):
    c = focus.AttentionConfig(Hq, Hkv, D, causal, scale, reserved, *strides)
    c = ctypes.byref(c) if cfg else None
    if which == "fwd":
        return L.focus_attention_fwd(c, q, k, v, dt, Tq, Tk, cu_q, cu_k, n, O, lse, ws, size, None)
    return L.focus_attention_bwd(c, dO, q, k, v, O, lse, dt, Tq, Tk, cu_q, cu_k, n, dq, B, B, ws, size, None)


@pytest.mark.parametrize("which", ["fwd", "bwd"])
def test_attention_checks(L, cpu_only, which):
    F = focus
    off = ctypes.c_void_p((1 << 20) + 8)
    for status, kw in ((F.ERR_NULL, {"cfg": False}), (F.ERR_CONFIG, {"causal": 2}), (F.ERR_CONFIG, {"scale": float("nan")}),
                       (F.ERR_CONFIG, {"reserved": 1}), (F.ERR_SHAPE, {"Hq": 3}), (F.ERR_SHAPE, {"Hq": 0}),
                       (F.ERR_SHAPE, {"Hkv": 0}), (F.ERR_SHAPE, {"Hq": 65536, "Hkv": 1}), (F.ERR_SHAPE, {"D": 0}),
                       (F.ERR_SHAPE, {"D": 60}), (F.ERR_SHAPE, {"D": 136}), (F.ERR_SHAPE, {"Tq": -1}),
                       (F.ERR_SHAPE, {"Tk": (1 << 30) + 1}), (F.ERR_SHAPE, {"n": -1}),
                       (F.ERR_SHAPE, {"strides": (128, 0, 0, 0, 0, 0)}), (F.ERR_SHAPE, {"strides": (0, 132, 0, 0, 0, 0)}),
                       (F.ERR_SHAPE, {"strides": (0, 0, 0, 0, 0, (1 << 24) + 8)}), (F.ERR_DTYPE, {"dt": 2}),
                       (F.ERR_NULL, {"q": None}), (F.ERR_NULL, {"v": None}), (F.ERR_NULL, {"O": None}),
                       (F.ERR_NULL, {"cu_q": B}), (F.ERR_NULL, {"cu_k": B}), (F.ERR_NULL, {"n": 2}), (F.ERR_SHAPE, {"k": off}),
                       (F.ERR_SHAPE, {"cu_q": B, "cu_k": ctypes.c_void_p((1 << 20) + 2)}), (F.ERR_WORKSPACE, {"ws": None}),
                       (F.ERR_WORKSPACE, {"size": 100}), (F.OK, {"cu_q": B, "cu_k": B, "n": 0})):
        assert attn(L, which, **kw) == status, kw
    if which == "bwd":
        assert attn(L, "bwd", lse=None) == F.ERR_NULL
        assert attn(L, "bwd", dO=None) == F.ERR_NULL
        assert attn(L, "bwd", dq=None) == F.ERR_NULL
    else:
        assert attn(L, "fwd", Tq=0, q=None, O=None) == F.OK


def test_attention_workspace(L):
    size = lambda call, D=128, Tq=64, Tk=64, n=1, **kw: L.focus_attention_workspace_size(
        call, ctypes.byref(focus.AttentionConfig(kw.get("Hq", 8), kw.get("Hkv", 2), D, 1, 0.1, 0, *(0,) * 6)), Tq, Tk, n)
    F = focus
    assert size(F.CALL_ATTENTION_FWD, Tq=1 << 20, Tk=1 << 20) == 256  # nothing to split
    # one query over many keys: partial outputs, maxima and sums of every part
    assert size(F.CALL_ATTENTION_FWD, Tq=1, Tk=8192) >= 256 + 2 * 8 * (128 + 2) * 4
    assert size(F.CALL_ATTENTION_BWD, Tq=1 << 16, Tk=1 << 16, n=32) >= 256 + 8 * (1 << 16) * 4
    for bad in (dict(D=12), dict(Tq=-1), dict(n=-1), dict(Hq=7)):
        assert size(F.CALL_ATTENTION_FWD, **bad) == 0
    assert size(F.CALL_NORM_FWD) == 0
    for Tq in (0, 1, 100, 1 << 20):
        for Tk in (0, 1, 100, 1 << 20):
            for n in (0, 1, 7, 1 << 20):
                for call in (F.CALL_ATTENTION_FWD, F.CALL_ATTENTION_BWD):
                    assert 256 <= size(call, Tq=Tq, Tk=Tk, n=n) < 1 << 34


def test_token_logprob_checks(L, cpu_only):
    F = focus

    def fwd(Z=B, dt=1, T=4, V=100, t=B, top=3, logp=B, ent=None, lse=B, tl=B, ti=B, ws=B, size=BIG):
        return L.focus_token_logprobs(Z, dt, T, V, t, top, logp, ent, lse, tl, ti, ws, size, None)

    def bwd(Z=B, dt=1, T=4, V=100, t=B, lse=B, ent=None, g=B, h=None, dZ=B, ws=B, size=BIG):
        return L.focus_token_logprobs_bwd(Z, dt, T, V, t, lse, ent, g, h, dZ, ws, size, None)

    odd = ctypes.c_void_p((1 << 20) + 1)
    for status, kw in ((F.ERR_DTYPE, {"dt": 3}), (F.ERR_CONFIG, {"top": 65}), (F.ERR_CONFIG, {"top": -1}), (F.ERR_SHAPE, {"V": 0}),
                       (F.ERR_SHAPE, {"T": -1}), (F.ERR_SHAPE, {"V": 1 << 31}), (F.ERR_NULL, {"Z": None}), (F.ERR_NULL, {"lse": None}),
                       (F.ERR_NULL, {"tl": None}), (F.ERR_NULL, {"ti": None}), (F.ERR_NULL, {"t": None}), (F.ERR_SHAPE, {"Z": odd}),
                       (F.ERR_SHAPE, {"t": ctypes.c_void_p((1 << 20) + 4)}), (F.ERR_WORKSPACE, {"size": 256}),
                       (F.OK, {"T": 0, "Z": None})):
        assert fwd(**kw) == status, kw
    for status, kw in ((F.ERR_DTYPE, {"dt": 3}), (F.ERR_SHAPE, {"V": 0}), (F.ERR_NULL, {"g": None}), (F.ERR_NULL, {"t": None}),
                       (F.ERR_NULL, {"h": B}), (F.ERR_NULL, {"dZ": None}), (F.ERR_SHAPE, {"dZ": odd}), (F.ERR_WORKSPACE, {"ws": None}),
                       (F.OK, {"T": 0})):
        assert bwd(**kw) == status, kw


def test_workspace_sizes(L):
    F = focus
    q = None
    assert L.focus_workspace_size(F.CALL_NORM_FWD, q, 10, 0, 64) == 256
    sizes = [F.norm_workspace_size(T, 2560) for T in (0, 1, 3, 4, 5, 100, 4096, 65536, 1 << 20)]
    assert sizes == sorted(sizes) and sizes[-1] == 256 + 1024 * 2560 * 8  # one for more tokens serves fewer
    assert F.norm_workspace_size(-1, 64) == 0 and F.norm_workspace_size(1, (1 << 24) + 1) == 0
    assert F.token_logprobs_workspace_size(8, 1000, 65) == 0 and F.token_logprobs_workspace_size(8, 0, 1) == 0
    assert F.token_logprobs_workspace_size(1, 1000, 5) == F.token_logprobs_workspace_size(100000, 1000, 5)
    assert L.focus_workspace_size(F.CALL_TOKEN_LOGPROBS_BWD, q, 8, 1000, 0) == 256


def test_attention_sizes_of_a_launch(L, cpu_only):
    """Work-items of a launch stay below 2^32: sizes past that are refused, sizes just below are not."""
    size = lambda Hq, Hkv, Tq, Tk, n: L.focus_attention_workspace_size(
        focus.CALL_ATTENTION_FWD, ctypes.byref(focus.AttentionConfig(Hq, Hkv, 8, 1, 0.1, 0, *(0,) * 6)), Tq, Tk, n)
    assert size(1, 1, 1 << 29, 1, 1) == 0 and size(1, 1, 1, 1 << 29, 1) == 0 and size(1, 1, (1 << 29) - 64, 1, 1) > 0
    assert size(64, 8, 1 << 25, 1, 1) == 0 and size(64, 8, (1 << 25) - 256, 1, 1) > 0
    assert size(64, 64, 1, 1 << 25, 1) == 0
    assert size(8, 8, 1, 1, 1 << 21) == 0 and size(8, 8, 1, 1, (1 << 21) - 1) > 0
    assert attn(L, "fwd", Hq=8, Hkv=8, cu_q=B, cu_k=B, n=1 << 21) == focus.ERR_SHAPE
