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


@pytest.mark.parametrize("top", [1, 5, 64])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("T,V", [(1, 131073), (9, 151935), (31, 140001), (40, 300001), (128, 280003)])
def test_rows_in_parts_with_ragged_ends(F, T, V, dt, top):
    """Parts that end inside a vector; the largest in one part or spread, equal over the parts; parts without a token."""
    from test_gpu_token_logprobs import check
    g = torch.Generator().manual_seed(V)
    i = torch.arange(V)
    kinds = [torch.randn(V, generator=g), torch.zeros(V), i.float() / 64, torch.where(i > V - 70, 3.0, -1.0),
             torch.where(i % 15000 == 0, 4.0, torch.randn(V, generator=g)), torch.where(i < V // 2, -math.inf, 1.0),
             torch.where(i == V - 1, 0.0, -math.inf), torch.full((V,), torch.finfo(DT[dt]).min)]
    announce(f"ragged parts {dt} {T}x{V} top={top}")
    Z = torch.stack([kinds[t % len(kinds)] for t in range(T)]).to(DT[dt]).cuda()
    t = torch.randint(-1, V, (T,), generator=g).cuda()
    check(F, Z, t, top)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_domain_errors_in_parts(F, bad):
    T, V = 5, 140001
    Z = (torch.randn(T, V, generator=torch.Generator().manual_seed(1)) * 2.5).bfloat16().cuda()
    Z[1, V - 2] = bad
    ws = F.workspace(F.token_logprobs_workspace_size(T, V, 3))
    logp, _, lse, _, _ = F.token_logprobs(Z, torch.zeros(T, dtype=torch.int64).cuda(), 3, ws=ws)
    assert F.check_flags(ws) == F.ERR_DOMAIN
    keep = [0, 2, 3, 4]
    assert torch.isfinite(logp[keep]).all() and torch.isfinite(lse[keep]).all()
    Z[1, V - 2] = 0.0
    logp = F.token_logprobs(Z, torch.tensor([3, V, -5, 0, 1]).cuda(), ws=ws)[0]
    assert F.check_flags(ws) == F.ERR_DOMAIN and logp[1] == 0 and logp[2] == 0
