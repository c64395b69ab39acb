"""Host-side checks of the binding of norms, attention and token log probabilities."""
import torch

from paper_2608_01847_amd import focus


def test_a_given_workspace_is_never_replaced():
    """The domain flag is raised in the workspace that the call gets: a larger one in its place would take it along."""
    small = torch.zeros(256, dtype=torch.uint8)
    assert focus._sized(small, 1 << 20, "cpu") is small
    own = focus._sized(None, 1000, "cpu")
    assert own.numel() == 1000 and not own[:256].any()
    assert focus._sized(None, 0, "cpu").numel() == 256
