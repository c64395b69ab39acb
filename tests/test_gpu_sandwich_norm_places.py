"""GPU tests of focus_sandwich_norm_* with outputs over inputs where rows are no whole eights, and start anywhere: the same bits."""
import pytest
import torch

from gpu_common import announce, require_gpu
from test_gpu_sandwich_norm import DT, make

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def F():
    return require_gpu()


@pytest.mark.parametrize("T,C", [(37, 7), (130, 65), (21, 1001), (1100, 999), (9, 1027), (300, 2561), (5, 8181), (70, 8201)])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_outputs_over_inputs(F, T, C, dt):
    announce(f"sandwich in place, ragged {dt} T={T} C={C}")
    t = make(T, C, DT[dt], 8, "token", True)
    ws = F.workspace(F.sandwich_norm_workspace_size(T, C))
    args = dict(b_post=t["b_post"], b_pre=t["b_pre"], residual_scale=0.7, kind=F.NORM_LAYER, ws=ws)
    names = ("w_post", "w_pre", "b_post", "b_pre", "gate")
    Y, N, stats = F.sandwich_norm_fwd(t["X"], t["B"], t["w_post"], t["w_pre"], gate=t["gate"], **args)
    dX, dB, g = F.sandwich_norm_bwd(t["dN"], t["dY"], t["X"], t["B"], t["w_post"], t["w_pre"], stats, gate=t["gate"], **args)
    rows = ("X", "B", "gate", "dN", "dY")

    def copies():  # each behind 64 elements that stay as they are, and in front of as many
        c, around = {}, []
        for k in rows:
            flat = torch.full((T * C + 128,), 7.0, dtype=DT[dt], device="cuda")
            c[k] = flat[64:64 + T * C].view(T, C).copy_(t[k])
            around += [flat[:64], flat[64 + T * C:]]
        return c, around

    for place, other in (("X", "B"), ("B", "gate"), ("gate", "X")):
        c, around = copies()
        Y2, N2, s2 = F.sandwich_norm_fwd(c["X"], c["B"], t["w_post"], t["w_pre"], gate=c["gate"], out=c[place], n_out=c[other], **args)
        assert torch.equal(Y2, Y) and torch.equal(N2, N) and torch.equal(s2, stats), place
        assert all((x == 7).all() for x in around)
    for places in (("dN", "dY", "gate"), ("X", "B", "dN"), ("dY", "gate", "X"), ("gate", "X", "B"), ("B", "dN", "dY")):
        c, around = copies()
        dX2, dB2, g2 = F.sandwich_norm_bwd(c["dN"], c["dY"], c["X"], c["B"], t["w_post"], t["w_pre"], stats, gate=c["gate"],
                                           out=c[places[0]], b_out=c[places[1]], gate_out=c[places[2]], **args)
        assert torch.equal(dX2, dX) and torch.equal(dB2, dB), places
        assert all(torch.equal(g2[n], g[n]) for n in names), places
        assert all((x == 7).all() for x in around)
