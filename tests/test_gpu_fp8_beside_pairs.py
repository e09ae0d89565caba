"""Kernels that hold tensor memory and wait for other CTAs of their cluster, on two streams at once."""
import pytest

pytestmark = pytest.mark.gpu


def test_products_of_clusters_beside_the_tensor_pipe_ceiling():
    """The ceiling's pairs hold all tensor memory of an SM, the small tiles' clusters (two CTAs an SM) a part each: they must not meet on an SM."""
    import torch
    from paper_2503_06564_b200 import trdq
    gen = torch.Generator(device="cuda").manual_seed(3)
    M, N, K = 2, 2304, 8192
    assert trdq.trdq_kernel_choice(2, M, K, N) == "gemm_fp8_kernel<16>, 8 a cluster, 2 an SM"
    q = trdq.trdq_fp8_quantize(torch.randn((M, K), generator=gen, device="cuda").bfloat16())
    w = trdq.trdq_fp8_quantize_weights(torch.randn((N, K), generator=gen, device="cuda").bfloat16())
    want = trdq.trdq_fp8_linear(*q, *w)
    ops = trdq.trdq_measure_mma_ceiling(256)
    torch.cuda.synchronize()
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    got = []
    for _ in range(40):
        with torch.cuda.stream(one):
            assert trdq.trdq_measure_mma_ceiling(256) == ops
        with torch.cuda.stream(two):
            got += [trdq.trdq_fp8_linear(*q, *w) for _ in range(2)]
    torch.cuda.synchronize()
    assert all(torch.equal(y, want) for y in got)
    assert trdq.trdq_device_status() == 0
