"""Rows that are not finite on the block-scaled path."""
import numpy as np
import pytest

from test_gpu_fp8 import _rotation

pytestmark = pytest.mark.gpu
T = 300


def test_a_bad_row_is_bad_throughout():
    """A NaN or an infinity among a row's values makes its whole row of the product NaN, and no other row's."""
    import torch
    from paper_2503_06564_b200 import trdq
    gen = torch.Generator(device="cuda").manual_seed(8)
    for M, N, K in ((6, 256, 256), (300, 1040, 640)):
        x = torch.randn((M, K), generator=gen, device="cuda").bfloat16()
        w, sw = trdq.trdq_fp8_quantize_weights(torch.eye(max(N, K), dtype=torch.bfloat16, device="cuda")[:N, :K].contiguous())   # most products are with a zero
        x[1, 7], x[3, K - 1], x[4, 130] = float("nan"), float("inf"), -float("inf")
        bad = torch.zeros(M, dtype=torch.bool, device="cuda")
        bad[[1, 3, 4]] = True
        for rot in (None, _rotation(np.random.default_rng(2), K)[0]):
            y = trdq.trdq_fp8_linear(*trdq.trdq_fp8_quantize(x, rot, T), w, sw)
            assert bool(y[bad].isnan().all()) and bool(y[~bad].isfinite().all())
        r, codes, scales = trdq.trdq_gated_norm_fp8(None, 0, x)
        y = trdq.trdq_fp8_linear(codes, scales, w, sw)
        assert bool(y[bad].isnan().all()) and bool(y[~bad].isfinite().all())
