"""Host-side checks of the workspace of the linear cross entropy: near what the call lays out in it, and never smaller for more tokens."""
import pytest

from paper_2608_01847_amd import focus

MB = 1 << 20


@pytest.fixture(scope="module")
def F():
    if not focus.LIBRARY.exists():
        pytest.skip("libfocus.so is not built")
    focus.lib()
    return focus


# One token: D and its transpose of a whole four of them in fp32, 2 x 2.3 MB, and 64 sums of one row each, 0.6. Otherwise X twice and dX (fp32), D and its transpose in
# fp32 (256 MiB at most), and of split sums no more than are worth a launch: the sizes that the calls need are 23 (bf16) and 77 MB (fp32), 33
# and 157, with 6 to 43 MB of the rest.
@pytest.mark.parametrize("T,V,K,most", [(1, 151936, 2560, 6), (16, 151936, 2560, 40), (301, 5003, 1008, 96), (1500, 3001, 512, 208)])
def test_sizes(F, T, V, K, most):
    size = F.linear_ce_workspace_size(T, V, K)
    assert size <= most * MB, size / MB
    assert size >= T * K * 4


@pytest.mark.parametrize("V,K", [(1, 16), (255, 16), (5003, 1008), (32000, 2560), (151936, 64), (3001, 8192), (70000, 33)])
def test_more_tokens_take_no_less(F, V, K):
    sizes = [F.linear_ce_workspace_size(T, V, K) for T in list(range(0, 700)) + list(range(700, 20000, 37)) + [1 << 17, 1 << 20, 1 << 24]]
    assert sizes == sorted(sizes)
