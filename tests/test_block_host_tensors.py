"""Host tensors given to the block-scaled calls and the fused norms are refused as the calls' own error, with or without a device at hand."""
import pytest


def _tensors():
    import torch
    x = torch.zeros((4, 256), dtype=torch.bfloat16)
    q, sx = torch.zeros((4, 256), dtype=torch.uint8), torch.zeros((2, 4))
    w, sw = torch.zeros((32, 256), dtype=torch.uint8), torch.zeros((1, 2))
    return x, q, sx, w, sw


CALLS = {
    "trdq_fp8_quantize": lambda f, x, q, sx, w, sw: f(x),
    "trdq_fp8_quantize_weights": lambda f, x, q, sx, w, sw: f(x),
    "trdq_fp8_linear": lambda f, x, q, sx, w, sw: f(q, sx, w, sw),
    "trdq_gated_norm": lambda f, x, q, sx, w, sw: f(x, x),
    "trdq_gated_norm_fp8": lambda f, x, q, sx, w, sw: f(None, 0, x, x),
    "trdq_gated_norm_backward": lambda f, x, q, sx, w, sw: f(x, x, x),
}


@pytest.mark.parametrize("name", CALLS)
def test_host_tensors(name):
    from paper_2503_06564_b200 import build, trdq
    build.build()
    with pytest.raises(trdq.TrdqError) as e:
        CALLS[name](getattr(trdq, name), *_tensors())
    assert e.value.status == 10 and name in str(e.value)
