"""What the product's self-test refuses, found on the host: no device is needed, and no pointer here is ever read."""
import pytest

NULL, SHAPE, ALIGN = 1, 2, 3
P = 1 << 20


@pytest.mark.parametrize("change, status", [
    (dict(M=-1), SHAPE), (dict(N=40), SHAPE), (dict(K=192), SHAPE), (dict(codes=None), NULL), (dict(sw=None), NULL), (dict(Y=None), NULL), (dict(ldy=40), SHAPE),
    (dict(ldy=52), ALIGN), (dict(w=P + 8), ALIGN), (dict(M=0, codes=None, Y=None), 0)])
def test_fp8_linear_expiry(change, status):
    from paper_2503_06564_b200 import build, trdq
    build.build()
    a = dict(codes=P, scales=P, M=5, K=256, w=P, sw=P, N=48, Y=P, ldy=48) | change
    assert trdq.lib().trdq_selftest_fp8_linear_expiry(a["codes"], a["scales"], a["M"], a["K"], a["w"], a["sw"], a["N"], a["Y"], a["ldy"], None) == status
