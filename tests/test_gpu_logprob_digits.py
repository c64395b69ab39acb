"""GPU tests of token log probabilities whose logits are large against their differences.

With m the row's largest logit, z - m is exact to 2^-24 of itself and log sum exp(z - m) good to 1e-5, whatever m is; a
log probability is their difference: 1e-5 + 2^-22 (|log p| + 1). The reference takes the same logits, in 64 bits, less m.
"""
import math

import pytest
import torch

from gpu_common import announce, require_gpu

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def F():
    return require_gpu()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("T,V", [(3, 1000), (2, 151936), (300, 5000)])
@pytest.mark.parametrize("offset", [0.0, 3e3, -1e5, 1e7, -3e30])
def test_log_probabilities_of_shifted_logits(F, T, V, dt, offset):
    announce(f"shifted logits {dt} T={T} V={V} offset={offset}")
    g = torch.Generator().manual_seed(V)
    step = max(1.0, abs(offset) * 2.0 ** (-7 if dt == "bf16" else -23))  # differences that the type holds there
    Z = (torch.randint(-8, 1, (T, V), generator=g) * step + offset).to(DT[dt])
    t = torch.randint(0, V, (T,), generator=g)
    logp, ent, lse, top_logp, top_index = F.token_logprobs(Z.cuda(), t.cuda(), 5)
    z = Z.double()
    lp = torch.log_softmax(z - z.amax(1, keepdim=True), 1)
    for got, ref in ((logp, lp.gather(1, t[:, None])[:, 0]), (top_logp, lp.gather(1, top_index.long().cpu()))):
        assert ((got.double().cpu() - ref).abs() <= 1e-5 + 2.0 ** -22 * (ref.abs() + 1)).all()
    assert ((lse.double().cpu() - torch.logsumexp(z, 1)).abs() <= 1e-5 + 2.0 ** -23 * abs(float(z.abs().max()))).all()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("T", [1, 300])
def test_rows_of_the_lowest_value(F, T, dt):
    """A row masked whole by the type's lowest value: every token is as likely as the next."""
    V = 90000
    Z = torch.full((T, V), torch.finfo(DT[dt]).min, dtype=DT[dt]).cuda()
    logp, ent, lse, top_logp, top_index = F.token_logprobs(Z, torch.full((T,), 17).cuda(), 3)
    for x in (-logp, ent, -top_logp):
        assert ((x - math.log(V)).abs() <= 1e-4).all()
    assert top_index.tolist() == [[0, 1, 2]] * T


def test_gradients_that_lse_has_no_digits_for(F):
    """Raise the domain flag; rows without a gradient of their own, masked whole or not, do not."""
    Z = torch.randn(6, 700).cuda()
    Z[1] += 7e4
    Z[2] -= 1e7
    Z[3] = torch.finfo(torch.float32).min
    Z[4] += 6e4
    Z[5] = -math.inf
    t = torch.zeros(6, dtype=torch.int64).cuda()
    ws = F.workspace(F.token_logprobs_workspace_size(6, 700))
    _, ent, lse, _, _ = F.token_logprobs(Z, t, ws=ws)
    assert F.check_flags(ws) == F.OK
    for row, far in ((0, False), (1, True), (2, True), (3, True), (4, False), (5, False)):
        for g, h in ((1.0, None), (None, 1.0), (0.0, 1.0), (0.0, 0.0)):
            d = [None if x is None else torch.zeros(6).cuda().index_fill_(0, torch.tensor([row]).cuda(), x) for x in (g, h)]
            dZ = F.token_logprobs_bwd(Z, t, lse, ent, *d, ws=ws)
            assert F.check_flags(ws) == (F.ERR_DOMAIN if far and (g or h) else F.OK), (row, g, h)
            keep = [i for i in range(6) if i != row]
            assert (dZ[keep] == 0).all()
    left_out = torch.full((6,), -1).cuda()
    F.token_logprobs_bwd(Z, left_out, lse, ent, torch.ones(6).cuda(), ws=ws)
    assert F.check_flags(ws) == F.OK
