"""GPU tests of focus_linear_ce_* on a workspace of the size that is asked for and no more, and on one made for more tokens."""
import pytest
import torch

from gpu_common import announce, require_gpu
from test_gpu_linear_ce import DT, make

pytestmark = pytest.mark.gpu

GUARD = 1 << 20


@pytest.fixture(scope="module")
def F():
    return require_gpu()


# one token, few; reductions long and short against the other sizes, so that products are split often, seldom and not at all; padded rows
SIZES = [(1, 20000, 256), (16, 5000, 64), (63, 40000, 16), (301, 5003, 1008), (1500, 3001, 512), (2000, 100, 64), (6000, 300, 96), (700, 2000, 1601),
         (513, 257, 1040)]


@pytest.mark.parametrize("T,V,K", SIZES)
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_nothing_behind_it_is_written(F, T, V, K, dt):
    announce(f"linear ce workspace {dt} T={T} V={V} K={K}")
    X, W, target, g, h = make(T, V, K, DT[dt], 5)
    size = F.linear_ce_workspace_size(T, V, K)
    whole = torch.full((size + GUARD,), 90, dtype=torch.uint8, device="cuda")
    ws = whole[:size]
    ws[:256] = 0
    logp, lse = F.linear_ce_fwd(X, W, target, ws=ws[:F.linear_ce_workspace_size(T, V, K, backward=False)])
    grads = F.linear_ce_bwd(X, W, target, lse, g, h, ws=ws)
    assert (whole[size:] == 90).all() and F.check_flags(ws) == F.OK
    more = F.workspace(F.linear_ce_workspace_size(2 * T + 77, V, K))
    more[256:] = 255
    assert all(torch.equal(a, b) for a, b in zip((logp, lse), F.linear_ce_fwd(X, W, target, ws=more)))
    assert all(torch.equal(a, b) for a, b in zip(grads, F.linear_ce_bwd(X, W, target, lse, g, h, ws=more)))
