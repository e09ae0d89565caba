"""The waits of the block-scaled product's CTA pairs run out and the kernel ends all the same.

In that kernel one warp waits for the accumulators with a time limit and passes the news on to the drain through hardware barriers, which have
none.  So both sides have to take part in every passage of a barrier, also after a wait has expired and the one warp no longer waits for
anything: the self-test leaves out the copies, every wait behind them expires, and all tiles of both sets of drain warps are gone through."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M, N, K", [
    (300, 256, 128),       # a tile a cluster, one k-block
    (256, 2048, 1152),     # a tile a cluster, nine k-blocks: accumulators are used a third time
    (5120, 2048, 1152),    # four or five tiles a cluster: both sets of drain warps, two or three tiles each
])
def test_the_pairs_end_without_their_operands(M, N, K):
    import torch
    from paper_2503_06564_b200 import trdq
    gen = torch.Generator(device="cuda").manual_seed(M)
    q, sx = trdq.trdq_fp8_quantize(torch.randn((M, K), generator=gen, device="cuda").bfloat16())
    qw, sw = trdq.trdq_fp8_quantize_weights(torch.randn((N, K), generator=gen, device="cuda").bfloat16())
    want = trdq.trdq_fp8_linear(q, sx, qw, sw)
    assert trdq.trdq_device_status() == 0
    trdq.trdq_selftest_fp8_linear_expiry(q, sx, qw, sw)
    word = trdq.trdq_device_status()   # synchronises
    # the MMAs' wait for operands always expires; what they then do without them may reach the warp that waits for accumulators before its own wait does
    assert word & 1 << 1 and word & ~(1 << 1 | 1 << 2) == 0
    assert trdq.trdq_device_status() == 0
    assert torch.equal(trdq.trdq_fp8_linear(q, sx, qw, sw), want)
