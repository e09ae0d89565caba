"""Block-scaled e4m3: the quantizers code by code and the product against sums in 64 bits."""
import numpy as np
import pytest

from oracle import trdq_oracle as O
from paper_2503_06564_b200 import workloads as WL
from util import to_dev_bf16

pytestmark = pytest.mark.gpu
TINY = np.float32(2.0 ** -100)


def _e4m3(v):
    """The nearest e4m3 number to fp32 values, ties to even, in double: 4 significant bits, spacing at least 2^-9, largest 448."""
    v = v.astype(np.float64)
    _, e = np.frexp(v)
    step = np.ldexp(1.0, np.maximum(e - 4, -9))
    return np.clip(np.rint(v / step) * step, -448.0, 448.0)


def _codes_of(v, top):
    """(values of the codes, scales) with the block maxima `top` broadcast against v; one fp32 rounding each as documented."""
    floor = np.maximum(top, TINY)
    mul = np.float32(448.0) * (np.float32(1.0) / floor)
    return _e4m3(v * mul), np.where(top > 0, floor * (np.float32(1.0) / np.float32(448.0)), np.float32(0)).astype(np.float32)


def _value(codes):
    import torch
    return codes.view(torch.float8_e4m3fn).float().cpu().numpy().astype(np.float64)


def _bits(rng, M, K, spread=True):
    x = rng.standard_normal((M, K))
    if spread:
        x *= np.exp(rng.uniform(-3, 3, (M, 1))) * np.where(rng.random(K) < 0.02, 30.0, 1.0)
    return WL.to_bf16_bits(x)


def _rotation(rng, K, groups=2):
    from paper_2503_06564_b200 import trdq
    signs = (rng.integers(0, 2, (groups, K)) * 2 - 1).astype(np.int8)
    smooth = np.exp(rng.uniform(-0.5, 0.5, (groups, K))).astype(np.float32)
    return trdq.Rotation(K, WL.group_bounds(groups), signs, smooth), signs, smooth


@pytest.mark.parametrize("M", [1, 2, 7, 8, 9, 31, 64, 257])
@pytest.mark.parametrize("K", [128, 256, 1152, 4096])
@pytest.mark.parametrize("rotated", [False, True])
def test_quantize_every_code(M, K, rotated):
    import torch
    from paper_2503_06564_b200 import trdq
    rng = np.random.default_rng(M * 10007 + K + rotated)
    bits = _bits(rng, M, K)
    bits[0, :128] = 0                                     # a block of zeros
    wide = np.zeros((M, K + 24), np.uint16)
    wide[:, :K] = bits
    x = to_dev_bf16(wide)[:, :K]
    for t in (100, 900):
        if rotated:
            rot, signs, smooth = _rotation(rng, K)
            g = rot.group_of(t)
            v = O.rotate(bits, O.fused_vectors(signs[g], smooth[g])[0])
        else:
            rot, v = None, WL.bf16_bits_to_f32(bits)
        codes, scales = trdq.trdq_fp8_quantize(x, rot, t)
        blocks = v.reshape(M, K // 128, 128)
        want, scale = _codes_of(blocks, np.abs(blocks).max(2, keepdims=True))
        assert codes.shape == (M, K) and scales.shape == (K // 128, M) and scales.dtype == torch.float32
        assert np.array_equal(_value(codes), want.reshape(M, K))
        assert np.array_equal(scales.cpu().numpy(), scale[:, :, 0].T)


@pytest.mark.parametrize("N", [16, 112, 128, 144, 1152])
@pytest.mark.parametrize("K", [128, 640])
@pytest.mark.parametrize("rotated", [False, True])
def test_weights_every_code(N, K, rotated):
    from paper_2503_06564_b200 import trdq
    rng = np.random.default_rng(N * 31 + K + rotated)
    bits = _bits(rng, N, K)
    rot, v = None, WL.bf16_bits_to_f32(bits)
    if rotated:
        rot, signs, smooth = _rotation(rng, K)
        v = O.rotate(bits, O.fused_vectors(signs[1], smooth[1])[1])
    codes, scales = trdq.trdq_fp8_quantize_weights(to_dev_bf16(bits), rot, 700)
    assert scales.shape == (-(-N // 128), K // 128)
    for i in range(-(-N // 128)):
        rows = slice(128 * i, min(N, 128 * i + 128))
        blocks = v[rows].reshape(-1, K // 128, 128)
        want, scale = _codes_of(blocks, np.abs(blocks).max((0, 2), keepdims=True))
        assert np.array_equal(_value(codes[rows]), want.reshape(-1, K))
        assert np.array_equal(scales[i].cpu().numpy(), scale[0, :, 0])


def test_quantize_extremes():
    """Subnormal, tiny and huge blocks; NaN and infinities stay in their own row."""
    import torch
    from paper_2503_06564_b200 import trdq
    x = torch.zeros((6, 256), dtype=torch.bfloat16, device="cuda")
    x[0, 0], x[1, :] = 1e-39, 2.0 ** -110
    x[2, 5], x[2, 6] = 3.3e38, -3.3e38
    x[3, 7], x[4, 130] = float("nan"), float("inf")
    x[5, :] = 1.0
    codes, scales = trdq.trdq_fp8_quantize(x)
    value, scales = _value(codes), scales.cpu().numpy()
    assert np.isfinite(value[[0, 1, 2, 5]]).all() and np.isfinite(scales[:, [0, 1, 2, 5]]).all()
    assert value[2, 5] == 448 and value[2, 6] == -448
    assert (value[1] == _e4m3(np.float32(2.0 ** -110) * (np.float32(448) * (np.float32(1) / TINY)) * np.ones(256, np.float32))).all()
    assert (value[5] == 448).all() and (scales[:, 5] == np.float32(1) / np.float32(448)).all()
    w, sw = trdq.trdq_fp8_quantize_weights(torch.eye(256, dtype=torch.bfloat16, device="cuda"))
    y = trdq.trdq_fp8_linear(codes, torch.from_numpy(scales).cuda(), w, sw).float().cpu().numpy()
    assert np.isnan(y[3]).any() and np.isnan(y[4]).any() and np.isfinite(y[[0, 1, 2, 5]]).all() and (y[5] == 1).all()


def _random_codes(gen, rows, cols):
    """e4m3 codes of every magnitude (no NaN)."""
    import torch
    c = torch.randint(0, 256, (rows, cols), generator=gen, device="cuda", dtype=torch.int32)
    c = torch.where((c & 0x7F) == 0x7F, c - 1, c)
    return c.to(torch.uint8).view(torch.float8_e4m3fn)


def _check_linear(M, N, K, act=0, bias=True, pad=0, seed=0):
    import torch
    from paper_2503_06564_b200 import trdq
    gen = torch.Generator(device="cuda").manual_seed(seed)
    q, qw = _random_codes(gen, M, K), _random_codes(gen, N, K)
    sx = torch.rand((K // 128, M), generator=gen, device="cuda") * 2e-3
    sw = torch.rand((-(-N // 128), K // 128), generator=gen, device="cuda") * 2e-2
    sx[K // 256, M // 2] = 0.0
    b = (torch.randn(N, generator=gen, device="cuda") * 2).bfloat16() if bias else None
    out = torch.full((M + 1, N + pad), 7.0, dtype=torch.bfloat16, device="cuda")
    y = trdq.trdq_fp8_linear(q, sx, qw, sw, b, out[:M, :N], act)
    assert y.data_ptr() == out.data_ptr()
    again = trdq.trdq_fp8_linear(q, sx, qw, sw, b, None, act)
    a = q.float().double().view(M, -1, 128) * sx.double().t()[:, :, None]
    w = qw.float().double().view(N, -1, 128) * sw.double().repeat_interleave(128, 0)[:N, :, None]
    a, w = a.reshape(M, K), w.reshape(N, K)
    ref = a @ w.t()
    size = a.abs() @ w.abs().t()
    if b is not None:
        ref, size = ref + b.double(), size + b.double().abs()
    # 128 products are added in the tensor core, whose alignment may drop a unit of the last place of the largest term each time (2^-23);
    # then per block one rounding of the scale, one of the product-sum, and at most 8 + 1 further additions of CTA sums and bias (2^-24)
    tol = (128 * 2.0 ** -23 + (2 * K // 128 + 9) * 2.0 ** -24) * size
    if act:
        ref = 0.5 * ref * (1 + torch.tanh(0.7978845608028654 * (ref + 0.044715 * ref ** 3)))
        tol = 1.13 * tol + 4e-6 * ref.abs() + 2.0 ** -130   # its slope is below 1.13; the fp32 evaluation
    tol = tol + 2.0 ** -8 * (ref.abs() + tol)               # bf16
    err = (y.double() - ref).abs()
    assert bool((err <= tol).all()), f"{(err / tol).max().item():.3f} of the tolerance"
    assert torch.equal(y, again)
    assert bool((out[M] == 7).all()) and (pad == 0 or bool((out[:, N:] == 7).all())), "written outside the output"
    assert trdq.trdq_device_status() == 0


@pytest.mark.parametrize("M", [1, 2, 15, 16, 17, 32, 33, 64, 65, 127, 128, 129, 300])
@pytest.mark.parametrize("N, K", [(16, 128), (144, 128), (128, 1152), (1040, 640)])
def test_linear_few_rows(M, N, K):
    _check_linear(M, N, K, pad=8 * (M % 3), seed=M * N + K)


@pytest.mark.parametrize("M, N, K", [(1, 16384, 4096), (5, 256, 16384), (40, 9216, 2048), (100, 1152, 8192), (257, 4624, 1152), (1000, 1152, 1152), (2049, 2320, 256),
                                     (4096, 512, 384), (515, 8192, 128), (3000, 272, 4608)])
@pytest.mark.parametrize("act", [0, 1])
def test_linear_sizes(M, N, K, act):
    _check_linear(M, N, K, act, bias=act == 0, seed=M + N + K)


def test_linear_of_quantized_layers_matches_the_unquantized_product():
    """Rotated on both sides the product is the layer's own, up to the codes' rounding (2^-4 per value, averaging out)."""
    import torch
    from paper_2503_06564_b200 import trdq
    rng = np.random.default_rng(5)
    M, N, K = 200, 272, 1152
    x, w = to_dev_bf16(_bits(rng, M, K)), to_dev_bf16(WL.to_bf16_bits(rng.standard_normal((N, K)) * 0.02))
    rot = _rotation(rng, K)[0]
    for t in (3, 800):
        y = trdq.trdq_fp8_linear(*trdq.trdq_fp8_quantize(x, rot, t), *trdq.trdq_fp8_quantize_weights(w, rot, t)).double()
        ref = x.double() @ w.double().t()
        # each code is off by at most 2^-4 of its value, the product by less than 2 x 2^-4 of its norm even if none of it averaged out
        assert ((y - ref).norm() / ref.norm()).item() < 2 * 2.0 ** -4
    other = trdq.trdq_fp8_linear(*trdq.trdq_fp8_quantize(x, rot, 3), *trdq.trdq_fp8_quantize_weights(w, rot, 800)).double()
    assert ((other - ref).norm() / ref.norm()).item() > 0.5, "groups that do not belong together"


def test_no_rows():
    import torch
    from paper_2503_06564_b200 import trdq
    x = torch.empty((0, 256), dtype=torch.bfloat16, device="cuda")
    codes, scales = trdq.trdq_fp8_quantize(x)
    assert codes.shape == (0, 256) and scales.shape == (2, 0)
    w, sw = trdq.trdq_fp8_quantize_weights(torch.ones((32, 256), dtype=torch.bfloat16, device="cuda"))
    assert trdq.trdq_fp8_linear(codes, scales, w, sw).shape == (0, 32)


def test_refusals():
    import torch
    from paper_2503_06564_b200 import trdq
    rng = np.random.default_rng(1)
    x = torch.randn((4, 256), device="cuda").bfloat16()
    w, sw = trdq.trdq_fp8_quantize_weights(torch.randn((32, 256), device="cuda").bfloat16())
    codes, scales = trdq.trdq_fp8_quantize(x)
    rot = _rotation(rng, 128)[0]
    perm = np.arange(256, dtype=np.int32)[None]
    full = trdq.Rotation(256, [0, 1000], np.ones((1, 256), np.int8), perm=perm)
    right = _rotation(rng, 256)[0]
    for call, status in ((lambda: trdq.trdq_fp8_quantize(x, rot, 1), 10), (lambda: trdq.trdq_fp8_quantize(x, full, 1), 10),
                         (lambda: trdq.trdq_fp8_quantize(x, right, 1000), 4), (lambda: trdq.trdq_fp8_quantize(x[:, :200]), 2),
                         (lambda: trdq.trdq_fp8_quantize(x[:, 4:132]), 3), (lambda: trdq.trdq_fp8_quantize(x, codes=torch.empty_like(codes[:2])), 2),
                         (lambda: trdq.trdq_fp8_linear(codes, scales.t().contiguous(), w, sw), 2), (lambda: trdq.trdq_fp8_linear(codes, scales, w[:, :128].contiguous(), sw), 2),
                         (lambda: trdq.trdq_fp8_linear(codes, scales, w[:24], sw), 2), (lambda: trdq.trdq_fp8_linear(codes, scales, w, sw, act=3), 2),
                         (lambda: trdq.trdq_fp8_linear(codes, scales, w, sw, out=torch.empty((4, 64), dtype=torch.bfloat16, device="cuda")[:, 4:36]), 3),
                         (lambda: trdq.trdq_fp8_linear(codes.cpu(), scales, w, sw), 10)):
        with pytest.raises(trdq.TrdqError) as e:
            call()
        assert e.value.status == status
    for call in (lambda: trdq.trdq_fp8_quantize(x.float()), lambda: trdq.trdq_fp8_linear(codes.float(), scales, w, sw),
                 lambda: trdq.trdq_fp8_linear(codes, scales.double(), w, sw), lambda: trdq.trdq_fp8_linear(codes, scales, w.t().contiguous().t(), sw),
                 lambda: trdq.trdq_fp8_quantize(x.t().contiguous().t())):
        with pytest.raises(AssertionError):
            call()


@pytest.mark.parametrize("M, K", [(9501, 4096), (4800, 4096), (20005, 1152)])
@pytest.mark.parametrize("rotated", [False, True])
def test_quantize_many_rows_as_few(M, K, rotated):
    """A warp takes several steps of rows where there are many: the codes and scales are those of the same rows quantized a few at a time."""
    import torch
    from paper_2503_06564_b200 import trdq
    gen = torch.Generator(device="cuda").manual_seed(M + K)
    x = (torch.randn((M, K), generator=gen, device="cuda") * torch.exp(torch.randn((M, 1), generator=gen, device="cuda"))).bfloat16()
    rot = _rotation(np.random.default_rng(1), K)[0] if rotated else None
    codes, scales = trdq.trdq_fp8_quantize(x, rot, 200)
    for at in range(0, M, 509):
        few = trdq.trdq_fp8_quantize(x[at:at + 509], rot, 200)
        assert torch.equal(codes[at:at + 509].view(torch.uint8), few[0].view(torch.uint8)) and torch.equal(scales[:, at:at + 509], few[1])


@pytest.mark.parametrize("M, N, K", [(32, 16384, 128), (64, 16384, 256), (96, 16384, 512), (200, 16384, 128), (256, 1152, 4608), (9, 4608, 4608), (16, 160, 16384), (130, 1040, 2176),
                                     (600, 4096, 256)])
@pytest.mark.parametrize("act", [0, 1])
def test_linear_cuts(M, N, K, act):
    """One and two CTAs an SM, more tiles than fit, tiles whose channel blocks are shared by two to eight CTAs, blocks that do not divide evenly, and the first sizes of the pairs."""
    _check_linear(M, N, K, act, seed=M + N + K)
    _check_linear(M, N, K, act, pad=8, bias=False, seed=M * 3 + N + K)


def test_linear_of_a_bad_channel_and_a_bad_row():
    """A NaN in a weight's channel spoils that column and no other, one among a row's codes that row, with the activation too."""
    import torch
    from paper_2503_06564_b200 import trdq
    gen = torch.Generator(device="cuda").manual_seed(4)
    for M in (3, 40, 700):
        K, N = 1152, 1040
        x, w = torch.randn((M, K), generator=gen, device="cuda").bfloat16(), torch.randn((N, K), generator=gen, device="cuda").bfloat16()
        (q, sx), (qw, sw) = trdq.trdq_fp8_quantize(x), trdq.trdq_fp8_quantize_weights(w)
        for act in (0, 1):
            want = trdq.trdq_fp8_linear(q, sx, qw, sw, act=act)
            bad_q, bad_w = q.clone().view(torch.uint8), qw.clone().view(torch.uint8)
            bad_q[M // 2, 700] = 0x7F
            bad_w[517, 3] = 0xFF
            y = trdq.trdq_fp8_linear(bad_q.view(q.dtype), sx, bad_w.view(q.dtype), sw, act=act)
            spoilt = torch.zeros((M, N), dtype=torch.bool, device="cuda")
            spoilt[M // 2] = True
            spoilt[:, 517] = True
            assert torch.equal(y.isnan(), spoilt) and torch.equal(y[~spoilt], want[~spoilt])
