"""The block-scaled product in every form that it chooses among: the shape gets that form, and its numbers are right."""
import pytest

from test_gpu_fp8 import _check_linear

pytestmark = pytest.mark.gpu

PAIR = "gemm_fp8_pair_kernel"
# (tokens a tile, CTAs a cluster, CTAs an SM) on 148 SMs
FORMS = [
    ((16, 1, 1), 1, 16, 128), ((16, 1, 1), 16, 16384, 512), ((16, 1, 2), 2, 32768, 128), ((16, 2, 1), 1, 4608, 2048), ((16, 2, 2), 2, 16384, 8192),
    ((16, 4, 1), 2, 16, 1152), ((16, 4, 2), 1, 4608, 4096), ((16, 8, 1), 1, 16, 4096), ((16, 8, 2), 2, 2304, 8192),
    ((32, 1, 1), 1500, 144, 128), ((32, 1, 2), 65, 8192, 128), ((32, 2, 1), 65, 2048, 2048), ((32, 2, 2), 17, 16384, 4608), ((32, 4, 1), 700, 16, 1152),
    ((32, 4, 2), 65, 2048, 4096), ((32, 8, 1), 300, 16, 4096), ((32, 8, 2), 17, 2304, 8192),
    ((64, 1, 1), 65, 8192, 1152), ((64, 1, 2), 129, 8192, 128), ((64, 2, 1), 1500, 144, 4096), ((64, 4, 1), 1500, 16, 4608), ((64, 8, 1), 512, 16, 16384),
    ((64, 8, 2), 300, 2048, 65536),
    # few rows against a wide matrix, whose tiles are many rounds of the pairs: the rows decide
    ((16, 1, 2), 1, 65536, 1152), ((32, 1, 2), 17, 40000, 1152), ((64, 2, 2), 64, 49152, 4096), (PAIR, 128, 65536, 1152),
    (PAIR, 300, 4608, 384), (PAIR, 4096, 512, 384), (PAIR, 2057, 4624, 1152),
]


@pytest.mark.parametrize("form, M, N, K", FORMS)
def test_form(form, M, N, K):
    from paper_2503_06564_b200 import trdq
    want = form if form is PAIR else "gemm_fp8_kernel<%d>, %d a cluster, %d an SM" % form
    assert trdq.trdq_kernel_choice(2, M, K, N) == want
    _check_linear(M, N, K, seed=M + N + K)


def test_what_the_choice_refuses():
    from paper_2503_06564_b200 import trdq
    for M, K, N in ((0, 256, 32), (4, 200, 32), (4, 256, 0), (4, 256, 40), (4, 131200, 32)):
        with pytest.raises(trdq.TrdqError) as e:
            trdq.trdq_kernel_choice(2, M, K, N)
        assert e.value.status == 2
