"""GPU tests of the linear cross entropy, the norms around a block and the gradient clipping on tensors whose elements or bytes pass
32 bits.

Bounds: those of the tests at ordinary sizes. Cross entropy: lse and logp by 4 sqrt(K) 2^-24 of the largest logit (independent
roundings) plus 2^-20 and lse's own rounding; bf16 gradients by 3.9e-3 of their norm (their roundings' root mean square). Rows of the norms do
not depend on one another: the last ones have the same bits in a call of their own. A norm of n bf16 numbers is a sum of n exact
squares in fp64, off by n 2^-53 = 5e-7 of itself, the root by half of that.
"""
import math

import pytest
import torch

from gpu_common import announce, require_gpu

pytestmark = pytest.mark.gpu

BF = torch.bfloat16


@pytest.fixture(scope="module")
def F():
    return require_gpu()


@pytest.fixture(autouse=True)
def memory():
    yield
    torch.cuda.empty_cache()


def random_bf16(rows, cols, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    out = torch.empty(rows, cols, dtype=BF, device="cuda")
    for r in range(0, rows, 30000):
        out[r:r + 30000] = torch.randn(min(30000, rows - r), cols, generator=g, device="cuda") * scale
    return out


def cross_entropy(F, T, V, K, seed):
    X, W = random_bf16(T, K, seed), random_bf16(V, K, seed + 1, 2.0 / math.sqrt(K))
    g = torch.Generator(device="cuda").manual_seed(seed + 2)
    target = torch.randint(0, V, (T,), generator=g, device="cuda")
    target[-1] = V - 1
    w = torch.full((T,), -1.0 / T, device="cuda")
    logp, lse = F.linear_ce_fwd(X, W, target)
    dX, dW = F.linear_ce_bwd(X, W, target, lse, w)
    torch.cuda.synchronize()
    return X, W, target, w, logp, lse, dX, dW


def check_lse(lse, logp, z_max, rlse, rlogp, K):
    lim = 4.0 * math.sqrt(K) * 2.0 ** -24 * max(1.0, z_max) + 2.0 ** -20
    assert ((lse.double() - rlse).abs() <= lim + 2.0 ** -23 * rlse.abs()).all()
    assert ((logp.double() - rlogp).abs() <= 2 * lim + 2.0 ** -23 * rlogp.abs()).all()


def test_cross_entropy_of_many_weights(F):
    T, V, K = 40, 270001, 8192  # 4.4 GB of weights
    announce("linear ce, 4.4 GB of weights")
    X, W, target, w, logp, lse, dX, dW = cross_entropy(F, T, V, K, 1)
    x = X.double()
    z = torch.cat([x @ W[v:v + 15000].double().t() for v in range(0, V, 15000)], 1)
    rlse = torch.logsumexp(z, 1)
    check_lse(lse, logp, float(z.abs().max()), rlse, z.gather(1, target[:, None])[:, 0] - rlse, K)
    D = -w.double()[:, None] * (z - rlse[:, None]).exp()
    D[torch.arange(T, device="cuda"), target] += w.double()
    rdX, err, size = torch.zeros_like(x), 0.0, 0.0
    for v in range(0, V, 15000):
        part, here = D[:, v:v + 15000], W[v:v + 15000].double()
        rdX += part @ here
        ref = part.t() @ x
        err, size = err + float((dW[v:v + 15000].double() - ref).square().sum()), size + float(ref.square().sum())
        if v + 15000 >= V:
            assert float((dW[v:].double() - ref).norm() / ref.norm()) <= 3.9e-3
    assert math.sqrt(err / size) <= 3.9e-3
    assert float((dX.double() - rdX).norm() / rdX.norm()) <= 3.9e-3


def test_cross_entropy_of_many_tokens(F):
    T, V, K = 530001, 300, 4096  # 4.3 GB of hidden states; D of one 256-wide piece 271 MB
    announce("linear ce, 4.3 GB of hidden states")
    X, W, target, w, logp, lse, dX, dW = cross_entropy(F, T, V, K, 4)
    wd, rdW, err, size = W.double(), torch.zeros(V, K, dtype=torch.float64, device="cuda"), 0.0, 0.0
    for t in range(0, T, 40000):
        e = slice(t, min(T, t + 40000))
        x = X[e].double()
        z = x @ wd.t()
        rlse = torch.logsumexp(z, 1)
        check_lse(lse[e], logp[e], float(z.abs().max()), rlse, z.gather(1, target[e][:, None])[:, 0] - rlse, K)
        D = -w[e].double()[:, None] * (z - rlse[:, None]).exp()
        D[torch.arange(len(x), device="cuda"), target[e]] += w[e].double()
        rdW += D.t() @ x
        ref = D @ wd
        this = float((dX[e].double() - ref).square().sum()), float(ref.square().sum())
        assert math.sqrt(this[0] / this[1]) <= 3.9e-3, t
    assert float((dW.double() - rdW).norm() / rdW.norm()) <= 3.9e-3


@pytest.mark.parametrize("C,gate", [(8192, "token"), (96, "feature")])
def test_norms_of_many_rows(F, C, gate):
    T = (2 ** 31 // C) + 1003
    announce(f"sandwich norm {T} x {C}")
    X, B, dN = (random_bf16(T, C, 10 + i) for i in range(3))
    w1, w2 = (1.0 + 0.1 * random_bf16(1, C, 20 + i)[0] for i in range(2))
    gates = random_bf16(T, C, 30) if gate == "token" else random_bf16(1, C, 30)[0]
    call = dict(kind=F.NORM_RMS)
    n = 64
    small = slice(T - n, T)
    of = lambda s: dict(call, gate=gates[s].contiguous() if gate == "token" else gates)
    want = F.sandwich_norm_fwd(X[small].contiguous(), B[small].contiguous(), w1, w2, **of(small))
    back = F.sandwich_norm_bwd(dN[small].contiguous(), None, X[small].contiguous(), B[small].contiguous(), w1, w2, want[2], **of(small))
    Y, N, stats = F.sandwich_norm_fwd(X, B, w1, w2, **of(slice(None)))
    assert torch.equal(Y[small], want[0]) and torch.equal(N[small], want[1]) and torch.equal(stats[:, small], want[2])
    dX, dB, grads = F.sandwich_norm_bwd(dN, None, X, B, w1, w2, stats, **of(slice(None)), out=Y, b_out=N)
    assert torch.equal(dX[small], back[0]) and torch.equal(dB[small], back[1])
    if gate == "token":
        assert torch.equal(grads["gate"][small], back[2]["gate"])


def test_clipping_of_a_large_tensor(F):
    announce("clip 2^31 elements")
    big = random_bf16(2 ** 16, 2 ** 15, 40).flatten()
    grads = [big, random_bf16(1, 100003, 41).flatten()[3:].clone(), torch.randn(7, device="cuda")]
    before = [big[-8192:].clone(), grads[1].clone(), grads[2].clone()]
    want = math.sqrt(sum(float(big[i:i + 2 ** 28].double().square().sum()) for i in range(0, big.numel(), 2 ** 28)) +
                     sum(float(g.double().square().sum()) for g in before[1:]))
    norm = F.clip_grad_norm(grads, 3.0)
    assert abs(norm.item() - want) <= 5e-7 * want
    for got, b in zip((big[-8192:], grads[1], grads[2]), before):
        ref = b.double() * (3.0 / want)
        lim = (2.0 ** -23 + 5e-7 + (2.0 ** -8 if b.dtype == BF else 0.0)) * ref.abs()
        assert ((got.double() - ref).abs() <= lim + 2.0 ** -149).all()
