"""GPU tests of the workspaces of norms, attention and token log probabilities as the binding takes them."""
import pytest
import torch

from gpu_common import require_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def F():
    return require_gpu()


def test_too_small_a_workspace_is_refused(F):
    X, w = torch.randn(40, 64).cuda(), torch.ones(64).cuda()
    Y, _, mean, rstd = F.norm_fwd(X, w)
    few, many = torch.randn(3, 4, 64).bfloat16().cuda(), torch.randn(4096, 4, 64).bfloat16().cuda()
    O, lse = F.attention_fwd(few, many, many)
    Z, t = torch.randn(3, 90000).cuda(), torch.zeros(3, dtype=torch.int64).cuda()
    small, header = (torch.zeros(n, dtype=torch.uint8).cuda() for n in (255, 256))
    for call in (lambda: F.norm_fwd(X, w, ws=small), lambda: F.norm_bwd(X, X, w, mean, rstd, ws=header),
                 lambda: F.attention_fwd(few, many, many, ws=header),
                 lambda: F.attention_bwd(few, few, many, many, O, lse, ws=header),
                 lambda: F.token_logprobs(Z, t, 5, ws=header), lambda: F.token_logprobs_bwd(Z, t, Z[:, 0].contiguous(),
                                                                                            d_logp=Z[:, 1].contiguous(), ws=small)):
        with pytest.raises(F.FocusError) as e:
            call()
        assert e.value.status == F.ERR_WORKSPACE


def test_the_flag_is_raised_in_the_given_workspace(F):
    """Few queries take a larger workspace than many (their keys are split): one sized for those raises or serves."""
    many, few = torch.randn(4096, 8, 64).bfloat16().cuda(), torch.randn(8, 8, 64).bfloat16().cuda()
    bad, keys = torch.tensor([0, 9], dtype=torch.int32).cuda(), torch.tensor([0, 4096], dtype=torch.int32).cuda()
    call = lambda ws: F.attention_fwd(few, many, many, bad, keys, ws=ws, out=torch.zeros_like(few), lse=torch.zeros(8, 8).cuda())
    with pytest.raises(F.FocusError) as e:
        call(F.workspace(256))
    assert e.value.status == F.ERR_WORKSPACE
    ws = F.workspace(F.attention_workspace_size(few, many))
    call(ws)
    assert F.check_flags(ws) == F.ERR_DOMAIN


def test_fp32_attention_in_its_own_workspace(F):
    """What the size function gives does, on shapes whose bf16 sums are split, and memory behind it is not touched."""
    for Tq, Tk in ((1, 3000), (600, 600)):
        q, dO = (torch.randn(Tq, 4, 64).cuda() for _ in range(2))
        k, v = (torch.randn(Tk, 2, 64).cuda() for _ in range(2))
        need = F.attention_workspace_size(q, k)
        assert need < F.attention_workspace_size(q.bfloat16(), k.bfloat16())
        room = F.workspace(need + 4096)
        room[need:] = 0xA5
        O, lse = F.attention_fwd(q, k, v, ws=room[:256])
        got = F.attention_bwd(dO, q, k, v, O, lse, ws=room[:need])
        want = F.attention_bwd(dO, q, k, v, O, lse)
        assert all(torch.equal(a, b) for a, b in zip(got, want)) and (room[need:] == 0xA5).all()
        with pytest.raises(F.FocusError):
            F.attention_bwd(dO, q, k, v, O, lse, ws=room[:need - 1])
