"""What the block-scaled 8-bit float calls and the fused norms refuse, found on the host before anything is launched: no device is needed,
and no pointer here is ever read."""
import ctypes as C

import pytest

NULL, SHAPE, ALIGN, MISMATCH, NOMEM = 1, 2, 3, 10, 8
P = 1 << 20   # an aligned address that nobody reads


@pytest.fixture(scope="module")
def lib():
    from paper_2503_06564_b200 import build, trdq
    build.build()
    return trdq.lib()


@pytest.mark.parametrize("change, status", [
    (dict(M=-1), SHAPE), (dict(K=0), SHAPE), (dict(K=64), SHAPE), (dict(K=131200), SHAPE), (dict(X=None), NULL), (dict(codes=None), NULL),
    (dict(scales=None), NULL), (dict(ldx=128), SHAPE), (dict(ldx=260), ALIGN), (dict(X=P + 8), ALIGN), (dict(codes=P + 8), ALIGN),
    (dict(scales=P + 2), ALIGN), (dict(M=0, X=None, codes=None, scales=None), 0)])
def test_quantize(lib, change, status):
    a = dict(X=P, ldx=256, M=3, K=256, codes=P, scales=P) | change
    assert lib.trdq_fp8_quantize(None, 0, a["X"], a["ldx"], a["M"], a["K"], a["codes"], a["scales"], None) == status


@pytest.mark.parametrize("change, status", [
    (dict(N=0), SHAPE), (dict(N=24), SHAPE), (dict(N=-16), SHAPE), (dict(K=100), SHAPE), (dict(W=None), NULL), (dict(codes=None), NULL),
    (dict(scales=None), NULL), (dict(W=P + 2), ALIGN), (dict(codes=P + 4), ALIGN), (dict(scales=P + 1), ALIGN)])
def test_quantize_weights(lib, change, status):
    a = dict(W=P, N=48, K=256, codes=P, scales=P) | change
    assert lib.trdq_fp8_quantize_weights(None, 0, a["W"], a["N"], a["K"], a["codes"], a["scales"], None) == status


@pytest.mark.parametrize("change, status", [
    (dict(M=-1), SHAPE), (dict(N=40), SHAPE), (dict(N=0), SHAPE), (dict(K=192), SHAPE), (dict(act=2), SHAPE), (dict(act=-1), SHAPE), (dict(ldy=40), SHAPE),
    (dict(ldy=52), ALIGN), (dict(codes=None), NULL), (dict(scales=None), NULL), (dict(w=None), NULL), (dict(sw=None), NULL), (dict(Y=None), NULL),
    (dict(codes=P + 8), ALIGN), (dict(w=P + 8), ALIGN), (dict(Y=P + 8), ALIGN), (dict(bias=P + 2), ALIGN), (dict(scales=P + 2), ALIGN), (dict(sw=P + 2), ALIGN),
    (dict(M=0, codes=None, Y=None), 0)])
def test_linear(lib, change, status):
    a = dict(codes=P, scales=P, M=5, K=256, w=P, sw=P, N=48, bias=P, Y=P, ldy=48, act=0) | change
    assert lib.trdq_fp8_linear(a["codes"], a["scales"], a["M"], a["K"], a["w"], a["sw"], a["N"], a["bias"], a["Y"], a["ldy"], a["act"], None) == status


def _op(**change):
    from paper_2503_06564_b200 import trdq
    a = dict(M=4, D=64, rows_per_sample=2, norm=1, post_norm=0, stream_f32=0, eps=1e-6, res_scale=1.0, X=P, ldx=64, branch_bf16=P, ldb=64, gate_bf16=P,
             ld_gate=64, shift_bf16=P, ld_shift=64, scale_bf16=P, ld_scale=64, weight_bf16=P, post_weight_bf16=P) | change
    return trdq.GatedNormOp(*[a[name] for name, _ in trdq.GatedNormOp._fields_])


BAD_OPS = [
    (dict(M=-1), SHAPE), (dict(D=0), SHAPE), (dict(D=60), SHAPE), (dict(D=8200), SHAPE), (dict(rows_per_sample=0), SHAPE), (dict(norm=0), SHAPE),
    (dict(norm=3), SHAPE), (dict(post_norm=3), SHAPE), (dict(post_norm=-1), SHAPE), (dict(eps=-1.0), SHAPE), (dict(eps=float("nan")), SHAPE),
    (dict(eps=float("inf")), SHAPE), (dict(res_scale=float("inf")), SHAPE), (dict(X=None), NULL), (dict(branch_bf16=None), NULL),
    (dict(branch_bf16=None, gate_bf16=None, post_weight_bf16=None, post_norm=2), NULL), (dict(ldx=56), SHAPE), (dict(ldx=68), ALIGN), (dict(X=P + 8), ALIGN),
    (dict(ldb=48), SHAPE), (dict(branch_bf16=P + 2), ALIGN), (dict(ld_gate=8), SHAPE), (dict(ld_shift=66), ALIGN), (dict(scale_bf16=P + 4), ALIGN),
    (dict(weight_bf16=P + 8), ALIGN), (dict(post_weight_bf16=P + 8), ALIGN), (dict(stream_f32=1, ldx=66), ALIGN)]


@pytest.mark.parametrize("change, status", BAD_OPS)
def test_gated_norm_op(lib, change, status):
    op = C.byref(_op(**change))
    assert lib.trdq_gated_norm(op, P, 64, P, 64, None) == status
    assert lib.trdq_gated_norm_fp8(op, None, 0, P, 64, P, P, None) == status


def test_no_rows(lib):
    assert lib.trdq_gated_norm(C.byref(_op(M=0, X=None)), None, 0, None, 0, None) == 0
    assert lib.trdq_gated_norm_fp8(C.byref(_op(M=0, X=None, D=128)), None, 0, None, 0, None, None, None) == 0
    assert lib.trdq_gated_norm(C.byref(_op(M=0, D=60)), None, 0, None, 0, None) == SHAPE


def test_gated_norm_outputs(lib):
    op = C.byref(_op())
    assert lib.trdq_gated_norm(None, P, 64, P, 64, None) == NULL
    assert lib.trdq_gated_norm(op, P, 64, None, 64, None) == NULL
    assert lib.trdq_gated_norm(op, P, 56, P, 64, None) == SHAPE
    assert lib.trdq_gated_norm(op, P + 2, 64, P, 64, None) == ALIGN
    assert lib.trdq_gated_norm(op, P + 4096, 64, P, 60, None) == SHAPE
    assert lib.trdq_gated_norm(op, P + 4096, 64, P + 8, 64, None) == ALIGN
    assert lib.trdq_gated_norm(op, P, 72, P, 64, None) == SHAPE       # in place, but with another row stride
    assert lib.trdq_gated_norm_fp8(op, None, 0, P, 64, P, P, None) == SHAPE   # 64 channels are no block
    wide = C.byref(_op(D=128, ldx=128, ldb=128, ld_gate=128, ld_shift=128, ld_scale=128))
    assert lib.trdq_gated_norm_fp8(wide, None, 0, P, 128, None, P, None) == NULL
    assert lib.trdq_gated_norm_fp8(wide, None, 0, P, 128, P, None, None) == NULL
    assert lib.trdq_gated_norm_fp8(wide, None, 0, P, 128, P + 8, P, None) == ALIGN


def _backward(lib, op, **change):
    a = dict(dH=P, lddh=64, dR=P, lddr=64, dX=P, lddx=64, dB=P, lddb=64, dgate=P, dshift=P, dscale=P, dweight=P, dpost=P, ws=P, bytes=1 << 30) | change
    return lib.trdq_gated_norm_backward(C.byref(op), a["dH"], a["lddh"], a["dR"], a["lddr"], a["dX"], a["lddx"], a["dB"], a["lddb"], a["dgate"], a["dshift"],
                                        a["dscale"], a["dweight"], a["dpost"], a["ws"], a["bytes"], None)


@pytest.mark.parametrize("change, status", BAD_OPS)
def test_backward_op(lib, change, status):
    assert _backward(lib, _op(**change)) == status


@pytest.mark.parametrize("change, status", [
    (dict(dH=None), NULL), (dict(lddh=32), SHAPE), (dict(dH=P + 2), ALIGN), (dict(lddr=60), SHAPE), (dict(dR=P + 2), ALIGN), (dict(lddx=68), ALIGN),
    (dict(dB=P + 2), ALIGN), (dict(dgate=P + 2), ALIGN), (dict(ws=None), NULL), (dict(ws=P + 8), ALIGN), (dict(bytes=16), NOMEM), (dict(lddx=72), SHAPE)])
def test_backward_outputs(lib, change, status):
    assert _backward(lib, _op(), **change) == status


@pytest.mark.parametrize("missing, grad", [("gate_bf16", "dgate"), ("shift_bf16", "dshift"), ("scale_bf16", "dscale"), ("weight_bf16", "dweight"),
                                           ("post_weight_bf16", "dpost")])
def test_no_gradient_of_what_is_not_there(lib, missing, grad):
    assert _backward(lib, _op(**{missing: None})) == NULL


def test_backward_workspace(lib):
    n = C.c_uint64(0)
    for M, rps in ((1, 1), (7, 3), (16384, 256), (100000, 1), (2 ** 31 - 1, 2 ** 31 - 1)):
        assert lib.trdq_gated_norm_backward_workspace(C.byref(_op(M=M, rows_per_sample=rps)), C.byref(n)) == 0
        samples = -(-M // min(rps, M))
        # three planes of one row of 64 sums per run; at least a run a sample, none longer than the sample
        assert n.value % (3 * 64 * 4) == 0 and n.value >= samples * 3 * 64 * 4 and n.value <= (2 * samples + 4 * 148 * 16) * 3 * 64 * 4
    assert lib.trdq_gated_norm_backward_workspace(C.byref(_op(M=0)), C.byref(n)) == 0 and n.value == 0
    assert lib.trdq_gated_norm_backward_workspace(None, C.byref(n)) == NULL
    assert lib.trdq_gated_norm_backward_workspace(C.byref(_op(D=12)), C.byref(n)) == SHAPE
