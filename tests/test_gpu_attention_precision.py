"""GPU tests of the size of the bf16 attention gradients' errors.

A gradient cannot be better than its result's rounding to bf16, whose size is measured on the reference itself. dv and dk have one
more rounding, of the operand P or dS of the last product: independent and of the same size, 1.41 times together. dq has dS in 16
bits, and from 257 keys on what the forward's rounding of O leaves in rowsum(dO O). All are held to 1.5 times the rounding, which
the error of a delta that is not corrected passes at most lengths here. The reference is the definition in float64.
"""
import math

import pytest
import torch

from gpu_common import announce, require_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def F():
    return require_gpu()


def reference(q, k, v, dO, causal):
    """dq, dk, dv of one sequence in float64, head by head."""
    q, k, v, dO = (t.double().cpu().transpose(0, 1).contiguous() for t in (q, k, v, dO))
    group, scale = q.shape[0] // k.shape[0], q.shape[2] ** -0.5
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    for h in range(q.shape[0]):
        K, V = k[h // group], v[h // group]
        S = q[h] @ K.T * scale
        if causal:
            S = S.masked_fill(~torch.ones_like(S, dtype=torch.bool).tril(S.shape[1] - S.shape[0]), -math.inf)
        P = torch.softmax(S, 1)
        dP = dO[h] @ V.T
        dS = P * (dP - (P * dP).sum(1, keepdim=True))
        dq[h] = dS @ K * scale
        dk[h // group] += dS.T @ q[h] * scale
        dv[h // group] += P.T @ dO[h]
    return [t.transpose(0, 1) for t in (dq, dk, dv)]


CASES = [(4, 4, 64, 16, 128, True), (64, 64, 16, 4, 128, True), (200, 200, 8, 2, 40, True), (256, 256, 4, 4, 128, False),
         (300, 300, 8, 8, 64, False), (1000, 1000, 8, 2, 128, True), (2048, 2048, 4, 1, 128, True), (64, 1000, 8, 2, 64, True),
         (900, 900, 2, 1, 96, False)]


@pytest.mark.parametrize("Tq,Tk,Hq,Hkv,D,causal", CASES)
def test_gradients_keep_their_digits(F, Tq, Tk, Hq, Hkv, D, causal):
    announce(f"attention digits {Tq}x{Tk} heads={Hq}/{Hkv} D={D} causal={causal}")
    g = torch.Generator().manual_seed(Tq + D)
    rnd = lambda T, H, s: (torch.randn(T, H, D, generator=g) * s).bfloat16().cuda()
    q, k, v, dO = rnd(Tq, Hq, 1.5), rnd(Tk, Hkv, 1.2), rnd(Tk, Hkv, 1.0), rnd(Tq, Hq, 1.0)
    O, lse = F.attention_fwd(q, k, v, causal=causal)
    got = F.attention_bwd(dO, q, k, v, O, lse, causal=causal)
    for name, x, ref in zip(("dq", "dk", "dv"), got, reference(q, k, v, dO, causal)):
        rounding = float((ref.bfloat16().double() - ref).norm())
        assert float((x.double().cpu() - ref).norm()) <= 1.5 * rounding, name


def test_packed_sequences_keep_their_digits(F):
    """Short and long sequences of one call whose sums are split: the short ones are one part's."""
    lengths, Hq, Hkv, D = [1500, 3, 120, 1400, 60], 2, 1, 128
    e = [sum(lengths[:i]) for i in range(len(lengths) + 1)]
    g = torch.Generator().manual_seed(3)
    rnd = lambda H, s: (torch.randn(e[-1], H, D, generator=g) * s).bfloat16().cuda()
    q, k, v, dO = rnd(Hq, 1.5), rnd(Hkv, 1.2), rnd(Hkv, 1.0), rnd(Hq, 1.0)
    cu = torch.tensor(e, dtype=torch.int32).cuda()
    assert F.attention_workspace_size(q, k, len(lengths)) > 256 + 2 * e[-1] * Hq * D * 4  # dq in parts
    O, lse = F.attention_fwd(q, k, v, cu)
    got = F.attention_bwd(dO, q, k, v, O, lse, cu)
    for s in range(len(lengths)):
        at = slice(e[s], e[s + 1])
        for name, x, ref in zip(("dq", "dk", "dv"), got, reference(q[at], k[at], v[at], dO[at], True)):
            rounding = float((ref.bfloat16().double() - ref).norm())
            # few numbers: the ratio of two small samples
            assert float((x[at].double().cpu() - ref).norm()) <= (1.5 if lengths[s] > 50 else 2.0) * rounding, (s, name)
