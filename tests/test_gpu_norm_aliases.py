"""GPU tests of the norms' outputs written over their inputs, in each kernel: a wave per row, a workgroup per row (whole and
ragged vectors), rows read several times."""
import pytest
import torch

from gpu_common import announce, require_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def F():
    return require_gpu()


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("C", [96, 97, 2560, 2561, 16400])
def test_outputs_over_inputs(F, C, dt):
    announce(f"norm aliases {dt} C={C}")
    g = torch.Generator().manual_seed(C)
    X, R, dY, dR = (torch.randn(70, C, generator=g).to(dt).cuda() for _ in range(4))
    w, b = (torch.randn(C, generator=g).cuda() for _ in range(2))
    for kind in (F.NORM_LAYER, F.NORM_RMS):
        for residual in (None, R):
            Y, H, mean, rstd = F.norm_fwd(X, w, b, residual, kind)
            x = X.clone()  # Y in X's place
            Y2, H2, mean2, rstd2 = F.norm_fwd(x, w, b, residual, kind, out=x)
            assert Y2.data_ptr() == x.data_ptr() and torch.equal(Y, Y2) and torch.equal(rstd, rstd2)
            assert residual is None or torch.equal(H, H2)
            assert kind == F.NORM_RMS or torch.equal(mean, mean2)
        r = R.clone()  # H in the residual's place
        H2 = F.norm_fwd(X, w, b, r, kind, h_out=r)[1]
        assert H2.data_ptr() == r.data_ptr() and torch.equal(H, H2)
        grads = F.norm_bwd(dY, H, w, mean, rstd, dR, kind, want_bias=True)
        for name in ("dY", "dR"):
            t = {"dY": dY.clone(), "dR": dR.clone()}
            got = F.norm_bwd(t["dY"], H, w, mean, rstd, t["dR"], kind, want_bias=True, out=t[name])
            assert got[0].data_ptr() == t[name].data_ptr()
            assert all(torch.equal(x, y) for x, y in zip(grads, got))
