"""GPU tests of rows of logits that end inside a kernel's step of 16,384.

What a row lacks to a whole step takes part in nothing: a row is, bit for bit, the row that goes on to the step's end with
logits of probability 0 (finite ones, 500 below the others, whose terms are exactly 0 in fp32).
"""
import math

import pytest
import torch

from gpu_common import announce, require_gpu

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
STEP = 16384


@pytest.fixture(scope="module")
def F():
    return require_gpu()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 7, 8, 9, 1000, 4096, 4103, 16376, 16383, 20000, 32767])
def test_a_row_is_the_row_that_goes_on_with_nothing(F, n, dt):
    announce(f"row ends {dt} n={n}")
    T, V = 300, -(-n // STEP) * STEP
    g = torch.Generator().manual_seed(n)
    whole = torch.full((T, V), -500.0)
    whole[:, :n] = torch.randn(T, n, generator=g) * 2.5
    whole = whole.to(DT[dt]).cuda()
    t = torch.randint(0, n, (T,), generator=g).cuda()
    for top in (0, min(n, 5)):
        got, want = F.token_logprobs(whole[:, :n].contiguous(), t, top), F.token_logprobs(whole, t, top)
        assert all(a is None or torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("mask", ["inf", "lowest"])
@pytest.mark.parametrize("n", [3, 8, 21, 4099, 16387])
def test_masked_logits_at_the_end(F, n, mask, dt):
    """Masked logits in and before the row's last vector of eight, and nothing else in it."""
    low = -math.inf if mask == "inf" else torch.finfo(DT[dt]).min
    g = torch.Generator().manual_seed(n)
    for T in (2, 300):
        Z = (torch.randn(T, n, generator=g) * 2.5).to(DT[dt])
        Z[:, max(1, n - 11):] = low
        Z[1, :-1] = low
        Z[1, -1] = 2.0
        ws = F.workspace(F.token_logprobs_workspace_size(T, n))
        logp, ent, lse, _, _ = F.token_logprobs(Z.cuda(), torch.zeros(T, dtype=torch.int64).cuda(), ws=ws)
        assert F.check_flags(ws) == F.OK
        z = Z.double()
        lp = torch.log_softmax(z, 1)
        ref = -(lp.exp() * lp.clamp(min=-1e300)).sum(1)
        assert ((lse.double().cpu() - torch.logsumexp(z, 1)).abs() <= 2e-5).all()
        assert ((ent.double().cpu() - ref).abs() <= 4e-5 * (1 + ref)).all()
        some = torch.isfinite(lp[:, 0])
        assert ((logp.double().cpu() - lp[:, 0]).abs()[some] <= 2e-5 + 2.0 ** -22 * lp[some, 0].abs()).all()
        assert torch.equal(torch.isneginf(logp.cpu()), ~some)
