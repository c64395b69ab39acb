"""Host-side checks of the binding of norms, attention and token log probabilities."""
import pytest
import torch

from paper_2608_01847_amd import focus


def test_a_given_workspace_is_never_replaced():
    """The domain flag is raised in the workspace that the call gets: a larger one in its place would take it along."""
    small = torch.zeros(256, dtype=torch.uint8)
    assert focus._sized(small, 1 << 20, "cpu") is small
    own = focus._sized(None, 1000, "cpu")
    assert own.numel() == 1000 and not own[:256].any()
    assert focus._sized(None, 0, "cpu").numel() == 256


def test_fp32_attention_asks_for_what_it_uses():
    """The fp32 kernels have no parts: the header, and in the backward a number per query and head."""
    if not focus.LIBRARY.exists():
        pytest.skip("libfocus.so is not built")
    for Tq, Tk, n, Hq, Hkv in ((8192, 8192, 4, 64, 8), (16384, 16384, 1, 2, 1), (1, 8192, 1, 32, 8), (0, 5, 1, 4, 2)):
        q, k = (torch.empty(T, H, 128, device="meta") for T, H in ((Tq, Hq), (Tk, Hkv)))
        delta = -(-Tq * Hq * 4 // 256) * 256
        assert focus.attention_workspace_size(q, k, n) == 256 + delta
        assert focus.attention_workspace_size(q.bfloat16(), k.bfloat16(), n) >= 256 + delta


def test_tensors_of_a_gpu_that_is_not_the_current_one(monkeypatch):
    """The call's stream is the current GPU's: work on another's tensors would run there, in no order with theirs."""
    class On:
        def __init__(self, device):
            self.device_index = device

        def get_device(self):
            return self.device_index

    for current in (0, 1):
        monkeypatch.setattr(torch.cuda, "current_device", lambda: current)
        focus._one_gpu("call", On(current), On(current), None)
        for tensors in ((On(1 - current), On(1 - current)), (On(current), On(1 - current)), (On(1 - current), None), (On(-1),)):
            with pytest.raises(ValueError):
                focus._one_gpu("call", *tensors)
