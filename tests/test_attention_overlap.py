"""Host-side checks of attention outputs that share memory with inputs (no kernel is launched, no pointer dereferenced).

Rows of 4 heads of 64 in fp32 are 1,024 bytes for queries, of 2 heads 512 for keys.
"""
import ctypes

import pytest

from paper_2608_01847_amd import focus

T, WQ, WK = 10, 1024, 512
APART = {n: (i + 1) << 24 for i, n in enumerate(("q", "k", "v", "O", "dO", "dq", "dk", "dv", "lse", "ws"))}


@pytest.fixture(scope="module")
def L():
    if not focus.LIBRARY.exists():
        pytest.skip("libfocus.so is not built")
    import torch
    if torch.cuda.is_available():
        pytest.skip("argument-check tests run in the CPU suite only")
    return focus.lib()


def call(L, which, strides=(0,) * 6, Tq=T, Tk=T, **at):
    p = {n: ctypes.c_void_p(x) for n, x in {**APART, **at}.items()}
    c = ctypes.byref(focus.AttentionConfig(4, 2, 64, 1, 0.1, 0, *(s // 4 for s in strides)))
    big = 1 << 34
    if which == "fwd":
        return L.focus_attention_fwd(c, p["q"], p["k"], p["v"], 0, Tq, Tk, None, None, 1, p["O"], p["lse"], p["ws"], big, None)
    return L.focus_attention_bwd(c, p["dO"], p["q"], p["k"], p["v"], p["O"], p["lse"], 0, Tq, Tk, None, None, 1, p["dq"],
                                 p["dk"], p["dv"], p["ws"], big, None)


def refused(L, which, **kw):
    return call(L, which, **kw) == focus.ERR_SHAPE


def passes(L, which, **kw):
    """Every check passed: there is no GPU to launch on."""
    return call(L, which, **kw) == focus.ERR_HIP


def test_whole_tensors(L):
    assert passes(L, "fwd") and passes(L, "bwd")
    assert passes(L, "fwd", O=APART["q"])
    assert refused(L, "fwd", O=APART["k"]) and refused(L, "fwd", O=APART["v"])
    assert refused(L, "fwd", O=APART["q"], strides=(2 * WQ, 0, 0, 0, 0, 0))
    for out in ("dq", "dk", "dv"):
        for other in ("q", "k", "v", "O", "dO", "dq", "dk", "dv"):
            assert other == out or refused(L, "bwd", **{out: APART[other]}), (out, other)


def test_ends_of_tensors(L):
    for out, other, w in (("O", "q", WQ), ("O", "k", WK)):
        assert passes(L, "fwd", **{out: APART[other] + T * w}) and refused(L, "fwd", **{out: APART[other] + T * w - 16})
        assert passes(L, "fwd", **{out: APART[other] - T * WQ}) and refused(L, "fwd", **{out: APART[other] - T * WQ + 16})
    assert passes(L, "bwd", dk=APART["q"] + T * WQ) and refused(L, "bwd", dk=APART["q"] + T * WQ - 16)
    assert passes(L, "bwd", dq=APART["k"] + T * WK) and refused(L, "bwd", dq=APART["k"] + T * WK - 16)
    assert passes(L, "bwd", dv=APART["dk"] - T * WK) and refused(L, "bwd", dv=APART["dk"] - T * WK + 16)


def test_no_rows(L):
    assert passes(L, "bwd", Tk=0, dk=APART["q"], dv=APART["q"])
    assert passes(L, "fwd", Tk=0, O=APART["k"])


def test_slices_at_one_stride(L):
    s = WQ + 2 * WK
    base = APART["dq"]
    fused = dict(dq=base, dk=base + WQ, dv=base + WQ + WK)
    assert passes(L, "bwd", strides=(0, 0, 0, s, s, s), **fused)
    for name, at in fused.items():
        for by in (16, -16):
            assert refused(L, "bwd", strides=(0, 0, 0, s, s, s), **{**fused, name: at + by}), (name, by)
    # whole rows apart: the same slice of another row is the same memory, the slice next to it is not
    for rows in (-T - 3, -T, 1 - T, -4, 0, 4, T - 1, T, T + 3):
        at = base + rows * s
        assert refused(L, "bwd", strides=(0, 0, 0, s, s, s), dq=base, dk=at) == (abs(rows) < T), rows
        assert passes(L, "bwd", strides=(0, 0, 0, s, s, s), dq=base, dk=at + WQ), rows
    # gradients in the gaps of the inputs' rows
    wide = 2 * s
    q = APART["q"]
    inputs, grads = dict(q=q, k=q + WQ, v=q + WQ + WK), dict(dq=q + s, dk=q + s + WQ, dv=q + s + WQ + WK)
    assert passes(L, "bwd", strides=(wide,) * 6, **inputs, **grads)
    assert refused(L, "bwd", strides=(wide,) * 6, **inputs, **{**grads, "dv": q + WQ + WK + 2 * wide})


def test_slices_at_different_strides(L):
    s = 4 * WQ
    assert refused(L, "bwd", strides=(0, 0, 0, s, 2 * s, 0), dq=APART["dq"], dk=APART["dq"] + WQ)
    # one row has no stride
    assert passes(L, "bwd", strides=(0, 0, 0, s, 2 * s, 0), dq=APART["dq"], dk=APART["dq"] + WQ, Tk=1)
    assert refused(L, "bwd", strides=(0, 0, 0, s, 2 * s, 0), dq=APART["dq"], dk=APART["dq"] + 2 * s, Tk=1)
    assert passes(L, "bwd", strides=(0, 0, 0, s, 2 * s, 0), dq=APART["dq"], dk=APART["dq"] + 2 * s + WQ, Tk=1)


def test_against_a_search(L):
    """Two tensors at one stride, at every offset of 16 bytes: what a walk over their rows finds."""
    s, Tq, Tk = WQ + WK, 3, 2
    rows = lambda base, n, w: {base + i * s + b for i in range(n) for b in range(0, w, 16)}
    a = rows(APART["dq"], Tq, WQ)
    for off in range(-3 * s, 4 * s, 16):
        shared = bool(a & rows(APART["dq"] + off, Tk, WK))
        assert refused(L, "bwd", strides=(0, 0, 0, s, s, 0), Tq=Tq, Tk=Tk, dk=APART["dq"] + off) == shared, off
