"""A sub-block on the block-scaled path stage by stage: what each call made of the codes, scales and sums that it really got, against 64 bits.

(The sub-block as a whole is compared with unquantized sums elsewhere, where the residual stream outweighs what the products add to it.)  u = 2^-24.
  quantizer: a code is half a step of e4m3 off (2^-4 of the value, at least 2^-10 of a scale), scale and factor four roundings; the rotation before it is a product and seven additions, 8 u of
    the block's sum of magnitudes, and passes on what its input is off by
  product: as in the tests of the product alone (128 products a block in the tensor core, 2^-23 of their magnitudes each; per block two fp32 roundings; sums of up to
    eight CTAs and the bias)"""
import numpy as np
import pytest

from oracle import trdq_oracle as O
from paper_2503_06564_b200 import workloads as WL
from test_gpu_fp8 import _bits
from test_gpu_gated_norm import EPS, U, _norm, _norm_tol, _rounded, _within
from util import to_dev_bf16

pytestmark = pytest.mark.gpu
T = 300


def _rotation_of(rng, K):
    """The handle, and the activations' and weights' vectors of T's group in double."""
    import torch
    from paper_2503_06564_b200 import trdq
    signs = (rng.integers(0, 2, (2, K)) * 2 - 1).astype(np.int8)
    smooth = np.exp(rng.uniform(-0.5, 0.5, (2, K))).astype(np.float32)
    rot = trdq.Rotation(K, WL.group_bounds(2), signs, smooth)
    g = rot.group_of(T)
    return rot, *(torch.from_numpy(np.ascontiguousarray(v)).cuda().double() for v in O.fused_vectors(signs[g], smooth[g]))


def _rotated(v, vec):
    """(v o vec) BlockDiag(H_128), and the blocks' sums of magnitudes."""
    import torch
    n = torch.arange(128, device="cuda")
    both = n[:, None] & n[None, :]
    H = 1.0 - 2.0 * (sum((both >> k) & 1 for k in range(7)) & 1)
    b = (v * vec).view(v.shape[0], -1, 128)
    size = b.abs().sum(2, keepdim=True).expand(b.shape)
    return (b @ H.double()).reshape(v.shape), size.reshape(v.shape)


def _values(codes, scales):
    return codes.float().double() * scales.double().t().repeat_interleave(128, 1)


def _weight_values(codes, scales):
    return codes.float().double() * scales.double().repeat_interleave(128, 0)[: codes.shape[0]].repeat_interleave(128, 1)


def _check_codes(codes, scales, v, tol):
    """tol: what v may be off by before the quantizer."""
    got = _values(codes, scales)
    step = 2.0 ** -10 * scales.double().t().repeat_interleave(128, 1)
    err, allowed = (got - v).abs(), tol + (2.0 ** -4 + 2.0 ** -22) * (v.abs() + tol) + step
    # the largest value becomes 448 whatever it is off by, and the scale with it
    assert bool((err <= allowed).all()), f"{(err / allowed).max().item():.3f} of the tolerance"


def _check_product(y, a, w, bias, gelu):
    import torch
    ref, size = a @ w.t(), a.abs() @ w.abs().t()
    if bias is not None:
        ref, size = ref + bias.double(), size + bias.double().abs()
    tol = (128 * 2.0 ** -23 + (2 * a.shape[1] // 128 + 9) * U) * size
    if gelu:
        ref = 0.5 * ref * (1 + torch.tanh(0.7978845608028654 * (ref + 0.044715 * ref ** 3)))
        tol = 1.13 * tol + 4e-6 * ref.abs() + 2.0 ** -130   # its slope is below 1.13; the fp32 evaluation
    _within(y, ref, _rounded(tol, ref, torch.bfloat16))


@pytest.mark.parametrize("M, width, rps", [(1, 1152, 1), (50, 384, 25), (517, 256, 100), (2100, 256, 2100)])
def test_every_stage_of_a_sub_block(M, width, rps):
    import torch
    from paper_2503_06564_b200 import trdq
    rng = np.random.default_rng(M + width)
    x, attn = to_dev_bf16(_bits(rng, M, width, False)), to_dev_bf16(_bits(rng, M, width, False))
    S = -(-M // rps)
    mod = to_dev_bf16(WL.to_bf16_bits(0.3 * rng.standard_normal((S, 6 * width))))
    part = [mod[:, i * width:(i + 1) * width] for i in range(6)]
    rows = torch.arange(M, device="cuda") // rps
    p = [v.double()[rows] for v in part]
    w1 = to_dev_bf16(WL.to_bf16_bits(rng.standard_normal((4 * width, width)) * 0.02))
    w2 = to_dev_bf16(WL.to_bf16_bits(rng.standard_normal((width, 4 * width)) * 0.02))
    b1 = to_dev_bf16(WL.to_bf16_bits(rng.standard_normal((1, 4 * width))))[0]
    (rot1, act1, wv1), (rot2, act2, wv2) = _rotation_of(rng, width), _rotation_of(rng, 4 * width)
    q1, q2 = trdq.trdq_fp8_quantize_weights(w1, rot1, T), trdq.trdq_fp8_quantize_weights(w2, rot2, T)
    for w, vec, (codes, scales) in ((w1, wv1, q1), (w2, wv2, q2)):
        v, size = _rotated(w.double(), vec)
        err = (_weight_values(codes, scales) - v).abs()
        step = 2.0 ** -10 * scales.double().repeat_interleave(128, 0)[: w.shape[0]].repeat_interleave(128, 1)
        assert bool((err <= 8 * U * size + (2.0 ** -4 + 2.0 ** -22) * (v.abs() + 8 * U * size) + step).all())

    def hidden(r, shift, scale):
        """LayerNorm and modulation of the stored r, and what fp32 may be off by."""
        n, tol = _norm(r.double(), "layer"), _norm_tol(r.double(), "layer")
        h = n * (1 + scale)
        tol = tol * (1 + scale).abs() + 6 * U * h.abs()
        return h + shift, tol + U * ((h + shift).abs() + shift.abs())

    # residual sum, norm and modulation, codes
    r, codes, scales = trdq.trdq_gated_norm_fp8(rot1, T, x, attn, gate=part[0], shift=part[1], scale=part[2], rows_per_sample=rps, eps=EPS)
    sum1 = x.double() + p[0] * attn.double()
    _within(r, sum1, _rounded(4 * U * (x.double().abs() + (p[0] * attn.double()).abs()), sum1, torch.bfloat16))
    h, h_tol = hidden(r, p[1], p[2])
    v, size = _rotated(h, act1)
    # the vector is multiplied into gain and shift before they are applied: two roundings more, of n (1 + scale) and of shift by themselves
    passed_on = _rotated(h_tol + 3 * U * ((h - p[1]).abs() + p[1].abs()), act1.abs())[1]
    _check_codes(codes, scales, v, passed_on + 8 * U * size)
    # first linear with GELU, its output as codes, second linear
    f = trdq.trdq_fp8_linear(codes, scales, *q1, b1, act=trdq.ACT_GELU_TANH)
    _check_product(f, _values(codes, scales), _weight_values(*q1), b1, True)
    codes2, scales2 = trdq.trdq_fp8_quantize(f, rot2, T)
    v, size = _rotated(f.double(), act2)
    _check_codes(codes2, scales2, v, 8 * U * size)
    y = trdq.trdq_fp8_linear(codes2, scales2, *q2)
    _check_product(y, _values(codes2, scales2), _weight_values(*q2), None, False)
    # y is the sub-block's output, not the codes' noise: without quantizers it is this, off by less than its own size
    exact = torch.nn.functional.gelu(h @ w1.double().t() + b1.double(), approximate="tanh") @ w2.double().t()
    assert torch.nn.functional.cosine_similarity(y.double().flatten(), exact.flatten(), 0).item() > 0.9
    # gate and residual, the next norm
    r2, h2 = trdq.trdq_gated_norm(r, y, gate=part[3], shift=part[4], scale=part[5], rows_per_sample=rps, eps=EPS)
    sum2 = r.double() + p[3] * y.double()
    _within(r2, sum2, _rounded(4 * U * (r.double().abs() + (p[3] * y.double()).abs()), sum2, torch.bfloat16))
    ref, tol = hidden(r2, p[4], p[5])
    _within(h2, ref, _rounded(tol, ref, torch.bfloat16))
    assert trdq.trdq_device_status() == 0
