"""The order of the tiles in the block-scaled product's largest calls."""
import pytest

from test_gpu_fp8 import _check_linear

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M", [7936, 7937, 8200, 9985])
def test_the_pairs_bands_of_tiles(M):
    """From 32 tiles of rows on the pairs go through them in bands of four, the last of which may be short: below that border, at it, and with last bands of one and of four."""
    from paper_2503_06564_b200 import trdq
    assert trdq.trdq_kernel_choice(2, M, 256, 400) == "gemm_fp8_pair_kernel"
    _check_linear(M, 400, 256, pad=8, seed=M)
