"""GPU tests of the digits that the gradients of focus_linear_ce_bwd keep with bf16 operands, against the definition in float64.

Bounds. Rounding D to bf16 moves every entry by half a step at most, 2^-8 of it, independently of the others, so that the norm of what it
costs a gradient is at most 2^-8 times the root of the sum over entries of (|D| times the norm of the row it is multiplied by)^2: `rounded`
below, over all entries but a token's target's. Of that entry the rest goes in too, rounded to bf16: 2^-8 of 2^-8 of it is left, the
same for all of its row. The weights of the tokens are scaled by powers of two, which rounds nothing. To that comes what a probability is off by (the logits'
and lse's errors, as in the tests of ordinary sizes) and 1e-5 for the sums. A gradient in bf16 is off by its own rounding besides: that of the
exact gradient, whose errors have the same distribution, and a twentieth for chance.

Before the target's rest went in, dW in fp32 was off by 1e-3 and more of its norm in these cases.
"""
import pytest
import torch

from gpu_common import announce, require_gpu
from test_gpu_linear_ce import make, reference, z_error

pytestmark = pytest.mark.gpu

BF = torch.bfloat16


@pytest.fixture(scope="module")
def F():
    return require_gpu()


def check(F, X, W, target, g, h=None, ws=None):
    K = X.shape[1]
    logp, lse = F.linear_ce_fwd(X, W, target, ws=ws)
    dX, dW = F.linear_ce_bwd(X, W, target, lse, g, h, dw_dtype=torch.float32, ws=ws)
    half = F.linear_ce_bwd(X, W, target, lse, g, h, ws=ws)[1]
    _, rlse, D, rdX, rdW, S = reference(X, W, target, g, h)
    p_err = 2 * (z_error(K, S) + 2.0 ** -20 + 2.0 ** -23 * float(rlse.abs().max()))
    others = D.square()
    kept = torch.nonzero(target >= 0)[:, 0]
    others[kept, target[kept]] = 0.0
    x2, w2 = X.double().square().sum(1), W.double().square().sum(1)
    for got, ref, rounded, what in ((dX, rdX, others @ w2, "dX"), (dW, rdW, others.t() @ x2, "dW"), (half, rdW, others.t() @ x2, "dW bf16")):
        size = float(ref.norm())
        lim = 2.0 ** -8 * float(rounded.sum().sqrt()) + (2.0 ** -16 + p_err + 1e-5) * size
        assert lim <= 7e-4 * size, (what, lim / size)  # far below what rounding every entry costs: the case shows it
        own = float((ref.to(BF).double() - ref).norm()) if got.dtype == BF else 0.0
        err = float((got.double() - ref).norm())
        assert err <= 1.05 * own + lim, (what, err / size, own / size, lim / size)


CASES = [(300, 5003, 1008), (700, 20000, 256), (64, 4000, 512), (5, 3000, 2560), (1, 5000, 256), (300, 5003, 1001), (9001, 3001, 192)]


@pytest.mark.parametrize("T,V,K", CASES)
@pytest.mark.parametrize("weights", ["mean", "own"])
def test_gradients_keep_their_digits(F, T, V, K, weights):
    announce(f"linear ce digits T={T} V={V} K={K} {weights}")
    X, W, target, g, _ = make(T, V, K, BF, T + V + K, ignored=0.1 if T > 1 else 0.0, spread=1.0)
    if weights == "mean":  # no power of two
        g = torch.full_like(g, -1.0 / (3 * T))
    ws = F.workspace(F.linear_ce_workspace_size(T, V, K))
    ws[256:] = 255
    check(F, X, W, target, g, ws=ws)
    assert F.check_flags(ws) == F.OK


def test_targets_that_many_tokens_share(F):
    # every token one of three targets, two of them neighbours: the rests of a tile are as many as its tokens
    T, V, K = 5003, 2000, 320
    announce("linear ce digits, shared targets")
    _, W, target, g, _ = make(T, V, K, BF, 41, spread=1.0)
    X = torch.randn(T, K, generator=torch.Generator().manual_seed(43)).to(BF).cuda()
    kept = target >= 0
    target[kept] = torch.tensor([255, 256, 1999], device="cuda")[torch.arange(int(kept.sum()), device="cuda") % 3]
    check(F, X, W, target, g)


def test_a_penalty_on_lse_beside_the_loss(F):
    announce("linear ce digits, lse penalty")
    X, W, target, g, h = make(600, 8000, 320, BF, 42, spread=1.0)
    check(F, X, W, target, g, 0.01 * h)


def test_several_pieces_of_the_vocabulary(F):
    # D of 40,000 tokens takes 512 MiB per 6,656 entries: the target's rest comes with its own piece, for dX with the last
    T, V, K = 40000, 21013, 32
    announce("linear ce digits, pieces")
    g = torch.Generator(device="cuda").manual_seed(3)
    X = torch.randn(T, K, generator=g, device="cuda").bfloat16()
    W = (0.15 * torch.randn(V, K, generator=g, device="cuda")).bfloat16()
    target = torch.randint(0, V, (T,), generator=g, device="cuda")
    w = -(0.2 + torch.rand(T, generator=g, device="cuda")) / T
    _, lse = F.linear_ce_fwd(X, W, target)
    dX, dW = F.linear_ce_bwd(X, W, target, lse, w, dw_dtype=torch.float32)
    rdW, rounded = torch.zeros(V, K, dtype=torch.float64, device="cuda"), 0.0
    for r in range(0, T, 8000):
        e = slice(r, r + 8000)
        _, rlse, D, rdX, part, S = reference(X[e], W, target[e], w[e], None)
        rdW += part
        D = D.square()
        D[torch.arange(8000, device="cuda"), target[e]] = 0.0
        rounded += float((D.sum(1) * X[e].double().square().sum(1)).sum())
        p_err = 2 * (z_error(K, S) + 2.0 ** -20 + 2.0 ** -23 * float(rlse.abs().max()))
        size, own = float(rdX.norm()), float((rdX.to(BF).double() - rdX).norm())
        lim = 2.0 ** -8 * float((D @ W.double().square().sum(1)).sum().sqrt()) + (2.0 ** -16 + p_err + 1e-5) * size
        err = float((dX[e].double() - rdX).norm())
        assert lim <= 7e-4 * size and err <= 1.05 * own + lim, (r, err / size, own / size, lim / size)
    size = float(rdW.norm())
    lim = 2.0 ** -8 * rounded ** 0.5 + (2.0 ** -16 + p_err + 1e-5) * size
    assert lim <= 7e-4 * size and float((dW.double() - rdW).norm()) <= lim, (float((dW.double() - rdW).norm()) / size, lim / size)
