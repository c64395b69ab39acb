"""GPU tests of the attention kernels whose sums are split into parts, at every width of head that has kernels of its own.

Reference and bounds are those of test_gpu_attention. The workspace is full of NaN past its header, so that a part which a
kernel does not write, or one that it reads without need, shows in the result.
"""
import pytest
import torch

from gpu_common import require_gpu
from test_gpu_attention import run_case

pytestmark = pytest.mark.gpu

HEADER = 256


class DirtyWorkspaces:
    """The binding with workspaces of 0xFF bytes (NaN in fp32) behind a cleared header."""

    def __init__(self, F):
        self.F = F

    def __getattr__(self, name):
        return getattr(self.F, name)

    def workspace(self, nbytes, device="cuda"):
        ws = self.F.workspace(nbytes, device)
        ws[HEADER:] = 0xFF
        return ws


@pytest.fixture(scope="module")
def F():
    return DirtyWorkspaces(require_gpu())


def sizes(F, lq, lk, Hq, Hkv, D):
    """Workspace bytes of the forward and the backward that the parts take."""
    import ctypes
    cfg = F.AttentionConfig(Hq, Hkv, D, 1, 1.0, 0, *(0,) * 6)
    size = lambda call: F.lib().focus_attention_workspace_size(call, ctypes.byref(cfg), sum(lq), sum(lk), len(lq))
    delta = -(-sum(lq) * Hq * 4 // 256) * 256
    return size(F.CALL_ATTENTION_FWD) - HEADER, size(F.CALL_ATTENTION_BWD) - HEADER - delta


@pytest.mark.parametrize("D", [8, 64, 72, 80, 96, 104, 128])
@pytest.mark.parametrize("causal", [True, False])
def test_two_sequences_in_parts(F, D, causal):
    for lengths, Hq in (([700, 301], 4), ([2200, 301], 2)):
        T = sum(lengths)
        fwd, bwd = sizes(F, lengths, lengths, Hq, 1, D)
        dq, dkv = T * Hq * D * 4, 2 * T * D * 4
        assert bwd >= 2 * dq + 2 * dkv and (fwd > 0 or Hq == 4)  # dq, dk with dv, the second one's forward: in two parts at least
        run_case(F, lengths, lengths, Hq, 1, D, "bf16", causal, seed=D)


@pytest.mark.parametrize("D", [64, 80, 128])
@pytest.mark.parametrize("causal", [True, False])
def test_few_queries_in_parts(F, D, causal):
    """Some parts hold no key that a query sees."""
    for lq, lk in (([3], [2000]), ([1, 1], [40, 1900]), ([0, 5], [600, 700])):
        assert sizes(F, lq, lk, 4, 2, D)[0] > 0
        run_case(F, lq, lk, 4, 2, D, "bf16", causal, seed=D)


@pytest.mark.parametrize("D", [40, 96, 128])
def test_no_parts(F, D):
    lengths = [70, 1, 0, 129]
    run_case(F, lengths, lengths, 4, 2, D, "bf16", True, seed=D)
    run_case(F, lengths, lengths, 4, 2, D, "f32", True, seed=D)


@pytest.mark.parametrize("scale", [0.02, 0.0, -0.1])
@pytest.mark.parametrize("D", [64, 96, 128])
def test_scales_of_both_signs(F, D, scale):
    """Also where v is read from LDS (from 65 features on) and the rows' statistics are divided by the scale."""
    for lengths in ([50], [900]):  # in one part, in several
        run_case(F, lengths, lengths, 2, 1, D, "bf16", True, seed=D, scale=scale)
    run_case(F, [50], [50], 2, 1, D, "f32", True, seed=D, scale=scale)


def test_parts_of_sequences_with_rows_before_and_behind(F):
    """Rows of no sequence have no parts: the join neither reads nor writes them."""
    T, a, b = 2400, 130, 2270
    cu = torch.tensor([a, 1300, b], dtype=torch.int32).cuda()
    g = torch.Generator().manual_seed(5)
    q, k, v, dO = (torch.randn(T, H, 80, generator=g).bfloat16().cuda() for H in (2, 1, 1, 2))
    ws = F.workspace(F.attention_workspace_size(q, k, 2))
    assert all(n > 0 for n in sizes(F, [T - 1, 1], [T - 1, 1], 2, 1, 80))
    O, lse = torch.full_like(q, 7.0), torch.full((2, T), 7.0).cuda()
    F.attention_fwd(q, k, v, cu, ws=ws, out=O, lse=lse)
    out = tuple(torch.full_like(t, 7.0) for t in (q, k, v))
    F.attention_bwd(dO, q, k, v, O, lse, cu, ws=ws, out=out)
    for x in (O, lse.t(), *out):
        assert (x[:a] == 7.0).all() and (x[b:] == 7.0).all() and torch.isfinite(x[a:b]).all()
    assert F.check_flags(ws) == F.OK


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("Tq,Tk", [(70, 70), (513, 513), (3, 2000)])
def test_output_in_the_queries_place(F, Tq, Tk, dt):
    g = torch.Generator().manual_seed(Tq)
    q, k, v = (torch.randn(T, H, 128, generator=g).to(dt).cuda() for T, H in ((Tq, 6), (Tk, 2), (Tk, 2)))
    O, lse = F.attention_fwd(q, k, v)
    x = q.clone()
    O2, lse2 = F.attention_fwd(x, k, v, out=x)
    assert O2.data_ptr() == x.data_ptr() and torch.equal(O, O2) and torch.equal(lse, lse2)


def test_outputs_over_other_inputs_are_refused(F):
    q, k, v, dO = (torch.randn(64, 2, 64).cuda() for _ in range(4))
    O, lse = F.attention_fwd(q, k, v)
    fresh = lambda: [torch.empty_like(q) for _ in range(3)]
    calls = [lambda: F.attention_fwd(q, k, v, out=k), lambda: F.attention_fwd(q, k, v, out=v)]
    for i in range(3):
        for t in (q, k, v, dO, O):
            out = fresh()
            out[i] = t
            calls.append(lambda out=tuple(out): F.attention_bwd(dO, q, k, v, O, lse, out=out))
    g = fresh()
    calls.append(lambda: F.attention_bwd(dO, q, k, v, O, lse, out=(g[0], g[1], g[1])))
    for call in calls:
        with pytest.raises(F.FocusError) as e:
            call()
        assert e.value.status == F.ERR_SHAPE
