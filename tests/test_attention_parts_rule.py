"""Host-side checks of which attention calls are split into parts, by the workspace that they ask for."""
import ctypes

import pytest

from paper_2608_01847_amd import focus


@pytest.fixture(scope="module")
def L():
    if not focus.LIBRARY.exists():
        pytest.skip("libfocus.so is not built")
    return focus.lib()


def fwd_parts(L, Hq, Hkv, Tq, Tk, n, D=128):
    cfg = focus.AttentionConfig(Hq, Hkv, D, 1, 0.1, 0, *(0,) * 6)
    size = L.focus_attention_workspace_size(focus.CALL_ATTENTION_FWD, ctypes.byref(cfg), Tq, Tk, n) - 256
    return max(1, size // (Tq * Hq * (D + 2) * 4))


@pytest.mark.parametrize("Hq,Hkv,T,n", [(32, 8, 256, 1), (32, 8, 512, 1), (8, 8, 512, 1), (8, 8, 1024, 1), (8, 8, 2048, 1), (4, 4, 2028, 4),
                                        (8, 2, 1800, 6)])
def test_short_prompts_stay_whole(L, Hq, Hkv, T, n):
    """The join of many rows costs more than their few tiles of keys take: in parts these took up to 2.5 times as long."""
    assert fwd_parts(L, Hq, Hkv, T, T, n) == 1


def test_few_rows_on_many_keys_are_split(L):
    assert fwd_parts(L, 32, 8, 1, 300, 1) == 1
    assert fwd_parts(L, 32, 8, 1, 1024, 1) >= 4 and fwd_parts(L, 32, 8, 1, 8192, 1) >= 32
    assert fwd_parts(L, 32, 8, 8, 8 * 4096, 8) >= 4
    assert fwd_parts(L, 2, 1, 2048, 2048, 1) >= 4 and fwd_parts(L, 2, 1, 4096, 4096, 1) >= 4
    assert fwd_parts(L, 8, 8, 256, 8192, 1) >= 8


def test_parts_are_never_more_than_the_join_takes(L):
    for Hq, Hkv in ((1, 1), (2, 1), (8, 8), (64, 8), (128, 1)):
        for Tq in (1, 7, 100, 1000, 5000):
            for Tk in (1, 64, 1000, 100000, 1 << 24):
                for n in (1, 3, 100):
                    assert fwd_parts(L, Hq, Hkv, Tq, Tk, n) <= 64


def key_parts(L, Hq, Hkv, Tq, Tk, n, D=128):
    """(parts of dq, parts of dk and dv; 0: whole) that add up to the workspace, which holds a whole fp32 tensor for each."""
    cfg = focus.AttentionConfig(Hq, Hkv, D, 1, 0.1, 0, *(0,) * 6)
    size = L.focus_attention_workspace_size(focus.CALL_ATTENTION_BWD, ctypes.byref(cfg), Tq, Tk, n) - 256
    whole = lambda n: -(-n * Tq * Hq * 4 // 256) * 256  # numbers of the rows: delta, and with dq's parts the sums of theirs
    dq, dkv = Tq * Hq * D * 4, 2 * Tk * Hkv * D * 4
    return [(q, k) for q in range(17) for k in range(17)
            if q != 1 and k != 1 and whole(1) + whole(q) + q * dq + k * dkv == size]


@pytest.mark.parametrize("Hq,Hkv,Tq,Tk,n,q", [(32, 8, 64, 2048, 1, 8), (4, 4, 512, 4096, 1, 16), (4, 4, 2028, 2028, 4, 0), (8, 8, 256, 256, 1, 0)])
def test_key_gradients_stay_whole_where_the_joins_cost_more(L, Hq, Hkv, Tq, Tk, n, q):
    """The joins go over every key, the saved tiles are of the queries: few queries on many keys took up to 1.35 times as long."""
    assert (q, 0) in key_parts(L, Hq, Hkv, Tq, Tk, n)


@pytest.mark.parametrize("Hq,Hkv,T,n,least", [(32, 8, 256, 1, 4), (2, 1, 4096, 1, 8), (8, 8, 1024, 1, 3), (64, 8, 8192, 4, 3), (4, 1, 8192, 1, 8)])
def test_key_gradients_of_few_workgroups_are_split(L, Hq, Hkv, T, n, least):
    assert max(k for q, k in key_parts(L, Hq, Hkv, T, T, n)) >= least
