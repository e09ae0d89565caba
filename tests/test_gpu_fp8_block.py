"""The block-scaled path as it is used: the calls of a sub-block after one another, captured and replayed, on another stream, two at once."""
import numpy as np
import pytest

from test_gpu_fp8 import _bits, _rotation
from util import to_dev_bf16
from paper_2503_06564_b200 import workloads as WL

pytestmark = pytest.mark.gpu


class _Mlp:
    """Gate and residual of the attention, norm and modulation, fc1 with GELU, fc2, gate and residual of the MLP with the next block's norm."""

    def __init__(self, M, width, rps, seed=0):
        import torch
        from paper_2503_06564_b200 import trdq
        rng = np.random.default_rng(seed)
        self.rps, self.t = rps, 300
        self.x, self.attn = to_dev_bf16(_bits(rng, M, width, False)), to_dev_bf16(_bits(rng, M, width, False))
        S = -(-M // rps)
        self.mod = to_dev_bf16(WL.to_bf16_bits(0.3 * rng.standard_normal((S, 6 * width))))
        self.w1 = to_dev_bf16(WL.to_bf16_bits(rng.standard_normal((4 * width, width)) * 0.02))
        self.w2 = to_dev_bf16(WL.to_bf16_bits(rng.standard_normal((width, 4 * width)) * 0.02))
        self.b1 = to_dev_bf16(WL.to_bf16_bits(rng.standard_normal((1, 4 * width))))[0]
        self.r1, self.r2 = _rotation(rng, width)[0], _rotation(rng, 4 * width)[0]
        self.q1, self.q2 = trdq.trdq_fp8_quantize_weights(self.w1, self.r1, self.t), trdq.trdq_fp8_quantize_weights(self.w2, self.r2, self.t)

    def part(self, i):
        width = self.x.shape[1]
        return self.mod[:, i * width:(i + 1) * width]

    def run(self):
        from paper_2503_06564_b200 import trdq
        given = dict(gate=self.part(0), shift=self.part(1), scale=self.part(2), rows_per_sample=self.rps)
        r, codes, scales = trdq.trdq_gated_norm_fp8(self.r1, self.t, self.x, self.attn, **given)
        h = trdq.trdq_fp8_linear(codes, scales, *self.q1, self.b1, act=trdq.ACT_GELU_TANH)
        y = trdq.trdq_fp8_linear(*trdq.trdq_fp8_quantize(h, self.r2, self.t), *self.q2)
        return trdq.trdq_gated_norm(r, y, gate=self.part(3), shift=self.part(4), scale=self.part(5), rows_per_sample=self.rps)

    def plain(self):
        """The same sub-block without any quantizer, in double."""
        import torch
        rows = torch.arange(self.x.shape[0], device="cuda") // self.rps
        p = lambda i: self.part(i).double()[rows]  # noqa: E731
        ln = lambda v: (v - v.mean(1, keepdim=True)) / (v.var(1, keepdim=True, unbiased=False) + 1e-6).sqrt()  # noqa: E731
        r = self.x.double() + self.attn.double() * p(0)
        h = (ln(r) * (1 + p(2)) + p(1)) @ self.w1.double().t() + self.b1.double()
        y = torch.nn.functional.gelu(h, approximate="tanh") @ self.w2.double().t()
        r2 = r + y * p(3)
        return r2, ln(r2) * (1 + p(5)) + p(4)


@pytest.mark.parametrize("M, width, rps", [(1, 1152, 1), (50, 384, 25), (517, 256, 100)])
def test_a_sub_block(M, width, rps):
    from paper_2503_06564_b200 import trdq
    block = _Mlp(M, width, rps)
    r, h = block.run()
    r_ref, h_ref = block.plain()
    # each product is off by less than 2 x 2^-4 of its norm (every code by at most 2^-4 of its value, both sides); GELU's slope is below 1.13, so y is off by less than
    # 2 x 1.13 x 2^-3 = 0.29 of what its norm would be without cancellation; r2 adds x, which is larger than y here
    assert ((r.double() - r_ref).norm() / r_ref.norm()).item() < 0.29
    assert ((h.double() - h_ref).norm() / h_ref.norm()).item() < 0.29
    assert trdq.trdq_device_status() == 0


def test_captured_and_replayed_with_new_inputs():
    import torch
    block, other = _Mlp(130, 256, 65), _Mlp(130, 256, 65, seed=7)
    want_first, want_second = block.run(), other.run()
    assert not torch.equal(want_first[1], want_second[1])
    other.q1, other.q2, other.r1, other.r2, other.b1 = block.q1, block.q2, block.r1, block.r2, block.b1
    want_second = other.run()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = block.run()
    graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(out, want_first))
    for name in ("x", "attn", "mod"):
        getattr(block, name).copy_(getattr(other, name))
    graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(out, want_second))


def test_two_streams_at_once():
    import torch
    blocks = [_Mlp(300, 384, 100, seed=s) for s in range(2)]
    want = [b.run() for b in blocks]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in blocks]
    got = [None, None]
    for _ in range(5):
        for i, (b, s) in enumerate(zip(blocks, streams)):
            with torch.cuda.stream(s):
                got[i] = b.run()
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert all(torch.equal(a, b) for a, b in zip(g, w))


def test_two_backward_passes_captured_side_by_side():
    """Each has a workspace of its own: replayed at once they give what each gives alone."""
    import torch
    from paper_2503_06564_b200 import trdq
    gen = torch.Generator(device="cuda").manual_seed(2)
    cases, graphs, outs, want = [], [], [], []
    for i in range(2):
        r, b, dh = (torch.randn((700, 640), generator=gen, device="cuda").bfloat16() for _ in range(3))
        w = torch.randn(640, generator=gen, device="cuda").bfloat16()
        mod = torch.randn((7, 640), generator=gen, device="cuda").bfloat16()
        call = lambda r=r, b=b, dh=dh, w=w, mod=mod: trdq.trdq_gated_norm_backward(r, b, dh, gate=mod, scale=mod, shift=mod, weight=w, rows_per_sample=100)  # noqa: E731
        want.append(call())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(call())
        graphs.append(graph)
        cases.append(call)
    streams = [torch.cuda.Stream() for _ in graphs]
    for _ in range(4):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for o, w in zip(outs, want):
        assert all(torch.equal(o[k], w[k]) for k in w if w[k] is not None)


def test_beside_the_int8_path():
    """The older calls before and after these on one stream, whose kernels start early, give what they give alone."""
    import torch
    from paper_2503_06564_b200 import trdq
    block = _Mlp(257, 256, 257)
    wts = trdq.trdq_prepare_weights(block.r1, block.w1, 8)
    r, h = block.run()
    y = trdq.trdq_linear(wts, block.t, *trdq.trdq_rotate_quantize(block.r1, block.t, h))
    torch.cuda.synchronize()
    for _ in range(3):
        r2, h2 = block.run()
        y2 = trdq.trdq_linear(wts, block.t, *trdq.trdq_rotate_quantize(block.r1, block.t, h2))
        assert torch.equal(r, r2) and torch.equal(h, h2) and torch.equal(y, y2)


@pytest.mark.parametrize("M", [0, 1, 2, 70])
def test_native_calls_and_the_general_way(M, monkeypatch):
    """Same outputs both ways, and every call has a native form for these arguments."""
    import torch
    from paper_2503_06564_b200 import trdq
    rng = np.random.default_rng(M)
    K = 256
    rot = _rotation(rng, K)[0]
    x = to_dev_bf16(_bits(rng, max(M, 1), K + 64))[:M]
    w = to_dev_bf16(_bits(rng, 48, K, False))
    mod = to_dev_bf16(_bits(rng, -(-M // 35) if M else 0, 3 * K, False)) if M else torch.empty((0, 3 * K), dtype=torch.bfloat16, device="cuda")
    gains = to_dev_bf16(_bits(rng, 1, K, False))[0]

    def calls():
        x2 = x[:, :K]
        codes, scales = trdq.trdq_fp8_quantize(x2)
        again = trdq.trdq_fp8_quantize(x[:, 64:], rot, 700, torch.empty_like(codes), torch.empty_like(scales))
        qw = trdq.trdq_fp8_quantize_weights(w, rot, 700)
        y = trdq.trdq_fp8_linear(codes.view(torch.uint8), scales, *qw, gains[:48])
        wide = torch.zeros((M, 64), dtype=torch.bfloat16, device="cuda")[:, :48]
        y2 = trdq.trdq_fp8_linear(codes, scales, *qw, None, wide, trdq.ACT_GELU_TANH)
        given = dict(gate=mod[:, :K], shift=mod[:, K:2 * K], scale=mod[:, 2 * K:], rows_per_sample=35, weight=gains, post_weight=gains, post_norm=trdq.NORM_RMS)
        r, h = trdq.trdq_gated_norm(x2, x[:, 64:], **given)
        r3, h3 = trdq.trdq_gated_norm(x2.float(), x[:, 64:], resid=torch.empty((M, K), device="cuda"), norm=trdq.NORM_RMS, res_scale=0.5)
        out = [codes, scales, *again, *qw, y, y2, r, h, r3, h3, *trdq.trdq_gated_norm_fp8(rot, 3, x2, x[:, 64:], **given), *trdq.trdq_gated_norm_fp8(None, 0, x2)]
        for g in (trdq.trdq_gated_norm_backward(r, x[:, 64:], h, **given), trdq.trdq_gated_norm_backward(r, None, h, r, res_scale=2.0)):
            out += [g[k] for k in ("dx", "db", "dgate", "dshift", "dscale", "dweight", "dpost_weight")]
        return out

    native = calls()
    taken = []

    class Declines:
        def __getattr__(self, name):
            return lambda *a: taken.append(name)

    with monkeypatch.context() as m:
        m.setattr(trdq, "_native", Declines())
        general = calls()
    assert set(taken) == {"fp8_quantize", "fp8_linear", "gated_norm", "gated_norm_fp8", "gated_norm_backward"}
    assert len(native) == len(general)
    for a, b in zip(native, general):
        assert (a is None) == (b is None)
        if a is None:
            continue
        assert a.dtype == b.dtype and a.shape == b.shape and a.stride() == b.stride()
        if a.dtype == torch.float8_e4m3fn:
            a, b = a.view(torch.uint8), b.view(torch.uint8)
        assert torch.equal(a, b)
    calls_of = trdq._calls()
    x2 = x[:, :K]
    assert calls_of.fp8_quantize(None, 0, x2, None, None, 0) is not None
    for left in (x2.float(), x2.cpu(), x2.t() if M > 1 else None, x2.half(), None, x2[0] if M else None):
        assert calls_of.fp8_quantize(None, 0, left, None, None, 0) is None


def test_a_closed_rotation_is_no_rotation_by_mistake():
    import torch
    from paper_2503_06564_b200 import trdq
    rot = _rotation(np.random.default_rng(0), 128)[0]
    x = torch.ones((2, 128), dtype=torch.bfloat16, device="cuda")
    rot.close()
    for call in (lambda: trdq.trdq_fp8_quantize(x, rot, 0), lambda: trdq.trdq_fp8_quantize_weights(x, rot, 0), lambda: trdq.trdq_gated_norm_fp8(rot, 0, x)):
        with pytest.raises(trdq.TrdqError) as e:
            call()
        assert e.value.status == 1
