"""GPU tests of focus_linear_ce_bwd in fp32 over several pieces of the vocabulary (D of 2,003 tokens takes 128 MiB per 16,640 entries).

Bounds as in the tests of ordinary sizes: p is off by what the logits and lse are, and a sum by 1e-5 of its terms' magnitudes.
"""
import pytest
import torch

from gpu_common import announce, require_gpu
from test_gpu_linear_ce import make, reference, z_error

pytestmark = pytest.mark.gpu

F32 = torch.float32


@pytest.fixture(scope="module")
def F():
    return require_gpu()


# three pieces, the last of another width; a last piece of five entries (tiles of 32 x 32); rows that are padded; a token count of whole fours
CASES = [(2003, 40013, 32), (2003, 16645, 48), (2003, 33281, 33), (4096, 20000, 64)]


@pytest.mark.parametrize("T,V,K", CASES)
def test_against_definition(F, T, V, K):
    announce(f"linear ce fp32 pieces T={T} V={V} K={K}")
    X, W, target, g, h = make(T, V, K, F32, T + V + K)
    target[:4] = torch.tensor([V - 1, 16639, 16640, 0])
    ws = F.workspace(F.linear_ce_workspace_size(T, V, K))
    ws[256:] = 255  # NaN
    logp, lse = F.linear_ce_fwd(X, W, target, ws=ws)
    ws[256:] = 255
    dX, dW = F.linear_ce_bwd(X, W, target, lse, g, h, ws=ws)
    assert F.check_flags(ws) == F.OK
    rlogp, rlse, D, rdX, rdW, S = reference(X, W, target, g, h)
    lim = z_error(K, S) + 2.0 ** -20
    assert ((lse.double() - rlse).abs() <= lim + 2.0 ** -23 * rlse.abs()).all()
    assert ((logp.double() - rlogp).abs() <= 2 * lim + 2.0 ** -23 * rlogp.abs()).all()
    terms = 2 * (lim + 2.0 ** -23 * float(rlse.abs().max())) + 1e-5
    D = D.abs()
    for got, ref, sizes, what in ((dX, rdX, D @ W.double().abs(), "dX"), (dW, rdW, D.t() @ X.double().abs(), "dW")):
        err = (got.double() - ref).abs()
        assert (err <= terms * sizes + 2.0 ** -24 * ref.abs() + 1e-30).all(), (what, float((err / sizes).max()), terms)
        assert float(err.norm()) <= terms * float(ref.norm())
    a = F.linear_ce_bwd(X, W, target, lse, g, h, want_dw=False, ws=ws)[0]
    b = F.linear_ce_bwd(X, W, target, lse, g, h, want_dx=False, ws=ws)[1]
    assert torch.equal(a, dX) and torch.equal(b, dW)


def test_tokens_without_a_gradient(F):
    announce("linear ce fp32 pieces, padding")
    T, V, K = 2003, 33000, 48
    X, W, target, g, _ = make(T, V, K, F32, 7)
    ws = F.workspace(F.linear_ce_workspace_size(T, V, K))
    lse = F.linear_ce_fwd(X, W, target, ws=ws)[1]
    want = F.linear_ce_bwd(X, W, target, lse, g, ws=ws)
    out = target < 0
    X[out], lse[out] = float("nan"), float("nan")
    got = F.linear_ce_bwd(X, W, target, lse, g, ws=ws)
    assert F.check_flags(ws) == F.OK and all(torch.equal(a, b) for a, b in zip(got, want)) and not got[0][out].any()
