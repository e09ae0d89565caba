"""Binding of ``libtrdq.so``: argument marshalling only.

Every function here has the name of the C entry point it calls (``include/trdq.h``)
and does nothing but turn torch tensors into pointers, sizes and the current
stream, in native code (``_calls``) for the hot calls on plain CUDA tensors, through ctypes otherwise and where the native
calls have not been built (with a warning).  All arithmetic runs in the CUDA kernels of the library; if ``libtrdq.so``
is missing the import of this module's library handle fails loudly, and there is no fallback for it of any kind.
"""
from __future__ import annotations

import ctypes as C
import importlib.util
import os
from functools import partial
from typing import Optional, Sequence, Tuple

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libtrdq.so")

OK = 0
STATUS_NAMES = {0: "TRDQ_OK", 1: "TRDQ_ERR_NULL", 2: "TRDQ_ERR_SHAPE", 3: "TRDQ_ERR_ALIGN", 4: "TRDQ_ERR_TIMESTEP",
                5: "TRDQ_ERR_GROUP", 6: "TRDQ_ERR_WBITS", 7: "TRDQ_ERR_CUDA", 8: "TRDQ_ERR_NOMEM", 9: "TRDQ_ERR_TIMEOUT",
                10: "TRDQ_ERR_MISMATCH", 11: "TRDQ_ERR_SCRATCH"}

EXPORTS = (
    "trdq_status_string", "trdq_version", "trdq_rotation_create", "trdq_rotation_destroy", "trdq_group_of",
    "trdq_find_group", "trdq_prepare_weights", "trdq_weights_destroy", "trdq_weights_info", "trdq_weights_view",
    "trdq_weights_export",
    "trdq_rotate_quantize", "trdq_linear", "trdq_linear_cfg", "trdq_gemm_i32", "trdq_device_status",
    "trdq_run_layers", "trdq_linear_splitk_workspace", "trdq_linear_splitk", "trdq_linear_splitk_static",
    "trdq_rotation_create_full", "trdq_zigzag_permutation", "trdq_rotate_quantize_asym", "trdq_linear_asym",
    "trdq_selftest_wait_expiry", "trdq_rotation_create_dense", "trdq_rotate_dense_workspace", "trdq_rotate_dense_quantize",
    "trdq_greedy_rotation_block", "trdq_linear_act", "trdq_norm_rotate_quantize", "trdq_kernel_choice",
    "trdq_measure_mma_ceiling", "trdq_fp8_quantize", "trdq_fp8_quantize_weights", "trdq_fp8_linear", "trdq_gated_norm", "trdq_gated_norm_fp8",
    "trdq_gated_norm_backward_workspace", "trdq_gated_norm_backward", "trdq_selftest_fp8_linear_expiry",
)


class TrdqError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = int(status)
        super().__init__(f"{where}: {STATUS_NAMES.get(self.status, self.status)} ({status_string(self.status)})")


class RotationSpec(C.Structure):
    _fields_ = [("K", C.c_int32), ("block", C.c_int32), ("num_groups", C.c_int32),
                ("t_bounds", C.POINTER(C.c_int32)), ("signs", C.POINTER(C.c_int8)), ("smooth", C.POINTER(C.c_float))]


class LayerOp(C.Structure):
    _fields_ = [("rot", C.c_void_p), ("w", C.c_void_p), ("X_bf16", C.c_void_p), ("ldx", C.c_int64), ("M", C.c_int32),
                ("codes", C.c_void_p), ("scales", C.c_void_p), ("bias_bf16", C.c_void_p), ("Y_bf16", C.c_void_p),
                ("ldy", C.c_int64), ("act", C.c_int32), ("workspace", C.c_void_p), ("workspace_bytes", C.c_uint64)]


class GatedNormOp(C.Structure):
    _fields_ = [("M", C.c_int32), ("D", C.c_int32), ("rows_per_sample", C.c_int32), ("norm", C.c_int32), ("post_norm", C.c_int32),
                ("stream_f32", C.c_int32), ("eps", C.c_float), ("res_scale", C.c_float), ("X", C.c_void_p), ("ldx", C.c_int64),
                ("branch_bf16", C.c_void_p), ("ldb", C.c_int64), ("gate_bf16", C.c_void_p), ("ld_gate", C.c_int64),
                ("shift_bf16", C.c_void_p), ("ld_shift", C.c_int64), ("scale_bf16", C.c_void_p), ("ld_scale", C.c_int64),
                ("weight_bf16", C.c_void_p), ("post_weight_bf16", C.c_void_p)]


_lib: Optional[C.CDLL] = None


def lib() -> C.CDLL:
    """The loaded library.  Raises if it has not been built: there is no other code path."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2503_06564_b200.build`")
        l = C.CDLL(LIB_PATH)
        l.trdq_status_string.restype = C.c_char_p
        l.trdq_status_string.argtypes = [C.c_int]
        l.trdq_version.restype = C.c_int32
        vp, i32, i64 = C.c_void_p, C.c_int32, C.c_int64
        l.trdq_rotation_create.argtypes = [C.POINTER(RotationSpec), C.POINTER(vp)]
        l.trdq_rotation_create_full.argtypes = [C.POINTER(RotationSpec), C.POINTER(i32), C.POINTER(C.c_int8), C.POINTER(vp)]
        l.trdq_zigzag_permutation.argtypes = [C.POINTER(C.c_float), i32, C.POINTER(i32)]
        l.trdq_rotation_destroy.argtypes = [vp]
        l.trdq_group_of.argtypes = [vp, i32, C.POINTER(i32)]
        l.trdq_find_group.argtypes = [C.POINTER(i32), i32, i32, C.POINTER(i32)]
        l.trdq_prepare_weights.argtypes = [vp, vp, i32, i32, C.POINTER(vp), vp]
        l.trdq_weights_destroy.argtypes = [vp]
        l.trdq_weights_info.argtypes = [vp, C.POINTER(i32), C.POINTER(i32), C.POINTER(i32), C.POINTER(i32)]
        l.trdq_weights_view.argtypes = [vp, i32, C.POINTER(vp), C.POINTER(vp)]
        l.trdq_weights_export.argtypes = [vp, i32, vp, vp, vp]
        l.trdq_rotate_quantize.argtypes = [vp, i32, vp, i64, i32, vp, vp, vp]
        l.trdq_linear.argtypes = [vp, i32, vp, vp, i32, vp, vp, i64, vp]
        l.trdq_norm_rotate_quantize.argtypes = [vp, i32, vp, i64, i32, vp, vp, i32, C.c_float, vp, vp, vp]
        l.trdq_linear_act.argtypes = [vp, i32, vp, vp, i32, vp, vp, i64, i32, vp]
        l.trdq_kernel_choice.argtypes = [i32, i32, i32, i32, i32, C.c_char_p, i32]
        l.trdq_measure_mma_ceiling.argtypes = [i32, C.POINTER(i32), vp]
        l.trdq_linear_cfg.argtypes = [vp, i32, C.POINTER(vp), C.POINTER(vp), C.POINTER(i32), vp, C.POINTER(vp),
                                      C.POINTER(i64), vp]
        l.trdq_gemm_i32.argtypes = [vp, i32, vp, i32, vp, i64, vp]
        l.trdq_run_layers.argtypes = [C.POINTER(LayerOp), i32, i32, vp]
        l.trdq_linear_splitk_workspace.argtypes = [vp, i32, C.POINTER(i32), C.POINTER(C.c_uint64)]
        l.trdq_linear_splitk.argtypes = [vp, i32, vp, vp, i32, vp, vp, i64, vp, C.c_uint64, vp]
        l.trdq_linear_splitk_static.argtypes = [vp, i32, vp, vp, i32, vp, vp, i64, vp]
        l.trdq_rotate_quantize_asym.argtypes = [vp, i32, vp, i64, i32, vp, vp, vp, vp]
        l.trdq_linear_asym.argtypes = [vp, i32, vp, vp, vp, i32, vp, vp, i64, vp]
        l.trdq_selftest_wait_expiry.argtypes = [vp]
        l.trdq_rotation_create_dense.argtypes = [i32, i32, C.POINTER(i32), C.POINTER(C.c_float), C.POINTER(C.c_float), C.POINTER(vp)]
        l.trdq_rotate_dense_workspace.argtypes = [vp, i32, C.POINTER(C.c_uint64)]
        l.trdq_rotate_dense_quantize.argtypes = [vp, i32, vp, i64, i32, vp, vp, vp, C.c_uint64, vp]
        l.trdq_greedy_rotation_block.argtypes = [C.POINTER(C.c_float), i32, i32, C.POINTER(C.c_double), C.POINTER(C.c_float),
                                                 C.POINTER(i32)]
        l.trdq_device_status.argtypes = [C.POINTER(C.c_uint32)]
        op = C.POINTER(GatedNormOp)
        l.trdq_fp8_quantize.argtypes = [vp, i32, vp, i64, i32, i32, vp, vp, vp]
        l.trdq_fp8_quantize_weights.argtypes = [vp, i32, vp, i32, i32, vp, vp, vp]
        l.trdq_fp8_linear.argtypes = [vp, vp, i32, i32, vp, vp, i32, vp, vp, i64, i32, vp]
        l.trdq_selftest_fp8_linear_expiry.argtypes = [vp, vp, i32, i32, vp, vp, i32, vp, i64, vp]
        l.trdq_gated_norm.argtypes = [op, vp, i64, vp, i64, vp]
        l.trdq_gated_norm_fp8.argtypes = [op, vp, i32, vp, i64, vp, vp, vp]
        l.trdq_gated_norm_backward_workspace.argtypes = [op, C.POINTER(C.c_uint64)]
        l.trdq_gated_norm_backward.argtypes = [op, vp, i64, vp, i64, vp, i64, vp, i64, vp, vp, vp, vp, vp, vp, C.c_uint64, vp]
        _lib = l
    return _lib


def status_string(status: int) -> str:
    return lib().trdq_status_string(int(status)).decode()


def _check(status: int, where: str) -> None:
    if status != OK:
        raise TrdqError(status, where)


_raw_stream = None


def _stream() -> int:
    """Handle of torch's current stream on the current device."""
    # The handle straight from torch's stream table: building a torch.cuda.Stream object around it costs 3.4 us a call,
    # this 0.2 us (of about 9 us that a binding call with given outputs took in all).
    global _raw_stream
    if _raw_stream is None:
        import torch
        torch.cuda.init()
        get, dev = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)
        _raw_stream = (lambda: get(dev())) if get and dev else (lambda: torch.cuda.current_stream().cuda_stream)
    return _raw_stream()


_native = None


class _GeneralWay:
    """Stands in for the native calls where they have not been built for the torch at hand: every call goes the general way."""

    def __getattr__(self, name):
        return lambda *args: None


def _calls():
    """The native form of the calls below (``csrc/calls.cpp``): it returns None for arguments it leaves to the general way."""
    global _native
    if _native is None:
        import warnings

        l = lib()
        try:
            from .build import calls_path
            spec = importlib.util.spec_from_file_location(f"{__package__}._calls", calls_path())   # (torch, whose libraries it needs, is loaded by now)
            native = importlib.util.module_from_spec(spec)
            spec.loader.exec_module(native)
            native.bind(*(C.cast(f, C.c_void_p).value for f in (
                l.trdq_rotate_quantize, l.trdq_norm_rotate_quantize, l.trdq_rotate_quantize_asym, l.trdq_linear_act, l.trdq_linear_cfg,
                l.trdq_linear_asym, l.trdq_linear_splitk_workspace, l.trdq_linear_splitk)))
            native.bind_block(*(C.cast(f, C.c_void_p).value for f in (
                l.trdq_fp8_quantize, l.trdq_fp8_quantize_weights, l.trdq_fp8_linear, l.trdq_gated_norm, l.trdq_gated_norm_fp8,
                l.trdq_gated_norm_backward_workspace, l.trdq_gated_norm_backward)))
        except ImportError as e:
            warnings.warn(f"the native calls cannot be used, calls take about twice the host time: {e}; build them with "
                          "`python -m paper_2503_06564_b200.build`")
            native = _GeneralWay()
        _native = native
    return _native


def _done(result, where: str):
    """The outputs of a native call, or its status as an exception."""
    if type(result) is int:
        raise TrdqError(result, where)
    return result


def _plain_empty(like):
    """new_empty of a tensor subclass would make one of its class; outputs are plain tensors."""
    import torch
    return partial(torch.empty, device=like.device)


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def trdq_find_group(t_bounds: Sequence[int], t: int) -> int:
    b = np.ascontiguousarray(t_bounds, dtype=np.int32)
    g = C.c_int32(-1)
    _check(lib().trdq_find_group(b.ctypes.data_as(C.POINTER(C.c_int32)), len(b) - 1, int(t), C.byref(g)), "trdq_find_group")
    return g.value


def trdq_zigzag_permutation(magnitude) -> np.ndarray:
    """Zigzag channel permutation (int32 [K]) from per-channel magnitudes; host only."""
    m = np.ascontiguousarray(magnitude, dtype=np.float32)
    perm = np.empty(m.shape[0], np.int32)
    _check(lib().trdq_zigzag_permutation(m.ctypes.data_as(C.POINTER(C.c_float)), int(m.shape[0]),
                                         perm.ctypes.data_as(C.POINTER(C.c_int32))), "trdq_zigzag_permutation")
    return perm


class Rotation:
    """Handle of a trdq_rotation (per-group device tables of one C_in)."""

    def __init__(self, K: int, t_bounds, signs, smooth=None, block: int = 128, perm=None, signs2=None):
        """perm (int32 [G][K]) selects the full transform of Eq. 9: rotation, zigzag permutation, second rotation
        (signs2: its +-1 vector, int8 [G][K] or None)."""
        self._h = C.c_void_p()
        b = np.ascontiguousarray(t_bounds, dtype=np.int32)
        s = np.ascontiguousarray(signs, dtype=np.int8)
        sm = None if smooth is None else np.ascontiguousarray(smooth, dtype=np.float32)
        spec = RotationSpec(int(K), int(block), int(len(b) - 1), b.ctypes.data_as(C.POINTER(C.c_int32)),
                            s.ctypes.data_as(C.POINTER(C.c_int8)),
                            None if sm is None else sm.ctypes.data_as(C.POINTER(C.c_float)))
        if perm is None:
            _check(lib().trdq_rotation_create(C.byref(spec), C.byref(self._h)), "trdq_rotation_create")
        else:
            pm = np.ascontiguousarray(perm, dtype=np.int32)
            s2 = None if signs2 is None else np.ascontiguousarray(signs2, dtype=np.int8)
            _check(lib().trdq_rotation_create_full(C.byref(spec), pm.ctypes.data_as(C.POINTER(C.c_int32)),
                                                   None if s2 is None else s2.ctypes.data_as(C.POINTER(C.c_int8)),
                                                   C.byref(self._h)), "trdq_rotation_create_full")
        self.K = int(K)
        self.num_groups = int(len(b) - 1)

    def group_of(self, t: int) -> int:
        g = C.c_int32(-1)
        _check(lib().trdq_group_of(self._h, int(t), C.byref(g)), "trdq_group_of")
        return g.value

    def close(self) -> None:
        if self._h:
            lib().trdq_rotation_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class DenseRotation(Rotation):
    """Handle of a trdq_rotation made of dense 128 x 128 blocks (Eq. 6-8): blocks fp32 [G][K/128][128][128]."""

    def __init__(self, K: int, t_bounds, blocks, smooth=None):
        self._h = C.c_void_p()
        b = np.ascontiguousarray(t_bounds, dtype=np.int32)
        G = int(len(b) - 1)
        blk = np.ascontiguousarray(blocks, dtype=np.float32)
        assert blk.shape == (G, int(K) // 128, 128, 128), blk.shape
        sm = None if smooth is None else np.ascontiguousarray(smooth, dtype=np.float32)
        _check(lib().trdq_rotation_create_dense(int(K), G, b.ctypes.data_as(C.POINTER(C.c_int32)),
                                                blk.ctypes.data_as(C.POINTER(C.c_float)),
                                                None if sm is None else sm.ctypes.data_as(C.POINTER(C.c_float)),
                                                C.byref(self._h)), "trdq_rotation_create_dense")
        self.K = int(K)
        self.num_groups = G


class Weights:
    """Handle of a trdq_weights (H_t(W) of one layer, quantized for every group)."""

    def __init__(self, handle: C.c_void_p):
        self._h = handle
        n, k, wb, g = C.c_int32(), C.c_int32(), C.c_int32(), C.c_int32()
        _check(lib().trdq_weights_info(self._h, C.byref(n), C.byref(k), C.byref(wb), C.byref(g)), "trdq_weights_info")
        self.N, self.K, self.wbits, self.num_groups = n.value, k.value, wb.value, g.value

    def view(self, g: int) -> Tuple[int, int]:
        """(device pointer of the codes, device pointer of the scales) of group g."""
        wq, sc = C.c_void_p(), C.c_void_p()
        _check(lib().trdq_weights_view(self._h, int(g), C.byref(wq), C.byref(sc)), "trdq_weights_view")
        return wq.value, sc.value

    def view_tensors(self, g: int):
        """Copies of group g's codes and scales as torch tensors (device)."""
        import torch
        if self.wbits == 8:
            codes = torch.empty((self.N, self.K), dtype=torch.int8, device="cuda")
            scales = torch.empty((self.N,), dtype=torch.float32, device="cuda")
        else:
            codes = torch.empty((self.N, self.K // 2), dtype=torch.uint8, device="cuda")
            scales = torch.empty((self.N, self.K // 128), dtype=torch.float32, device="cuda")
        _check(lib().trdq_weights_export(self._h, int(g), _ptr(codes), _ptr(scales), _stream()), "trdq_weights_export")
        return codes, scales

    def close(self) -> None:
        if self._h:
            lib().trdq_weights_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def trdq_prepare_weights(rot: Rotation, W_bf16, wbits: int = 8) -> Weights:
    assert W_bf16.is_cuda and W_bf16.is_contiguous() and W_bf16.dim() == 2 and W_bf16.element_size() == 2
    if W_bf16.shape[1] != rot.K:
        raise TrdqError(2, "trdq_prepare_weights (K of W differs from the rotation's)")
    h = C.c_void_p()
    _check(lib().trdq_prepare_weights(rot._h, _ptr(W_bf16), int(W_bf16.shape[0]), int(wbits), C.byref(h), _stream()),
           "trdq_prepare_weights")
    return Weights(h)


def trdq_rotate_quantize(rot: Rotation, t: int, X_bf16, codes=None, scales=None):
    """codes int8 [M,K], scales fp32 [M] of the rotated activations at time-step t."""
    done = (_native or _calls()).rotate_quantize(rot._h.value, rot.K, t, X_bf16, codes, scales)
    if done is not None:
        return _done(done, "trdq_rotate_quantize")
    import torch
    assert X_bf16.is_cuda and X_bf16.dim() == 2 and X_bf16.element_size() == 2 and X_bf16.stride(1) == 1
    M = int(X_bf16.shape[0])
    empty = X_bf16.new_empty if type(X_bf16) is torch.Tensor else _plain_empty(X_bf16)
    if codes is None:
        codes = empty((M, rot.K), dtype=torch.int8)
    if scales is None:
        scales = empty((M,), dtype=torch.float32)
    ldx = int(X_bf16.stride(0)) if M > 1 else rot.K
    _check(lib().trdq_rotate_quantize(rot._h, int(t), _ptr(X_bf16), ldx, M, _ptr(codes), _ptr(scales), _stream()),
           "trdq_rotate_quantize")
    return codes, scales


def trdq_norm_rotate_quantize(rot: Rotation, t: int, X_bf16, shift_bf16=None, scale_bf16=None, rows_per_sample: Optional[int] = None,
                              eps: float = 1e-6, codes=None, scales=None):
    """LayerNorm + per-sample modulation + rotation + per-token quantizer in one kernel."""
    done = (_native or _calls()).norm_rotate_quantize(rot._h.value, rot.K, t, X_bf16, shift_bf16, scale_bf16, rows_per_sample, eps, codes, scales)
    if done is not None:
        return _done(done, "trdq_norm_rotate_quantize")
    import torch
    assert X_bf16.is_cuda and X_bf16.dim() == 2 and X_bf16.element_size() == 2 and X_bf16.stride(1) == 1
    M = int(X_bf16.shape[0])
    if rows_per_sample is None:
        rows_per_sample = max(M, 1)
    empty = X_bf16.new_empty if type(X_bf16) is torch.Tensor else _plain_empty(X_bf16)
    if codes is None:
        codes = empty((M, rot.K), dtype=torch.int8)
    if scales is None:
        scales = empty((M,), dtype=torch.float32)
    ldx = int(X_bf16.stride(0)) if M > 1 else rot.K
    _check(lib().trdq_norm_rotate_quantize(rot._h, int(t), _ptr(X_bf16), ldx, M, _ptr(shift_bf16), _ptr(scale_bf16),
                                           int(rows_per_sample), float(eps), _ptr(codes), _ptr(scales), _stream()),
           "trdq_norm_rotate_quantize")
    return codes, scales


def trdq_rotate_dense_workspace(rot: Rotation, M: int) -> int:
    n = C.c_uint64(0)
    _check(lib().trdq_rotate_dense_workspace(rot._h, int(M), C.byref(n)), "trdq_rotate_dense_workspace")
    return int(n.value)


def trdq_rotate_dense_quantize(rot: Rotation, t: int, X_bf16, codes=None, scales=None, workspace=None):
    """codes int8 [M,K], scales fp32 [M] of the activations rotated by the dense blocks of time-step t."""
    import torch
    assert X_bf16.is_cuda and X_bf16.dim() == 2 and X_bf16.element_size() == 2 and X_bf16.stride(1) == 1
    M = int(X_bf16.shape[0])
    empty = X_bf16.new_empty if type(X_bf16) is torch.Tensor else _plain_empty(X_bf16)
    if codes is None:
        codes = empty((M, rot.K), dtype=torch.int8)
    if scales is None:
        scales = empty((M,), dtype=torch.float32)
    if workspace is None:
        workspace = empty((max(1, trdq_rotate_dense_workspace(rot, M)),), dtype=torch.uint8)
    ldx = int(X_bf16.stride(0)) if M > 1 else rot.K
    _check(lib().trdq_rotate_dense_quantize(rot._h, int(t), _ptr(X_bf16), ldx, M, _ptr(codes), _ptr(scales), _ptr(workspace),
                                            int(workspace.numel() * workspace.element_size()), _stream()),
           "trdq_rotate_dense_quantize")
    return codes, scales


def trdq_greedy_rotation_block(x_calib, gauss) -> Tuple[np.ndarray, int]:
    """(R fp32 [128,128], n) of Eq. 6-7 for one block; host only."""
    x = np.ascontiguousarray(x_calib, dtype=np.float32)
    g = np.ascontiguousarray(gauss, dtype=np.float64)
    assert x.ndim == 2 and x.shape[1] == 128 and g.ndim == 3 and g.shape[1:] == (128, 128)
    R = np.empty((128, 128), np.float32)
    n = C.c_int32(0)
    _check(lib().trdq_greedy_rotation_block(x.ctypes.data_as(C.POINTER(C.c_float)), int(x.shape[0]), int(g.shape[0]),
                                            g.ctypes.data_as(C.POINTER(C.c_double)), R.ctypes.data_as(C.POINTER(C.c_float)),
                                            C.byref(n)), "trdq_greedy_rotation_block")
    return R, int(n.value)


def trdq_linear(w: Weights, t: int, codes, scales, bias_bf16=None, out=None):
    """bf16 [M,N] output of the integer GEMM with the dequantizing epilogue."""
    done = (_native or _calls()).linear(w._h.value, w.N, t, codes, scales, bias_bf16, out, ACT_NONE)
    if done is not None:
        return _done(done, "trdq_linear")
    import torch
    M = int(codes.shape[0])
    empty = codes.new_empty if type(codes) is torch.Tensor else _plain_empty(codes)
    if out is None:
        out = empty((M, w.N), dtype=torch.bfloat16)
    ldy = int(out.stride(0)) if M > 1 else w.N
    _check(lib().trdq_linear(w._h, int(t), _ptr(codes), _ptr(scales), M, _ptr(bias_bf16), _ptr(out), ldy, _stream()),
           "trdq_linear")
    return out


ACT_NONE, ACT_GELU_TANH = 0, 1


def trdq_linear_act(w: Weights, t: int, codes, scales, bias_bf16=None, out=None, act: int = ACT_GELU_TANH):
    """trdq_linear with the following activation (GELU, tanh form) folded into the epilogue."""
    done = (_native or _calls()).linear(w._h.value, w.N, t, codes, scales, bias_bf16, out, act)
    if done is not None:
        return _done(done, "trdq_linear_act")
    import torch
    M = int(codes.shape[0])
    empty = codes.new_empty if type(codes) is torch.Tensor else _plain_empty(codes)
    if out is None:
        out = empty((M, w.N), dtype=torch.bfloat16)
    ldy = int(out.stride(0)) if M > 1 else w.N
    _check(lib().trdq_linear_act(w._h, int(t), _ptr(codes), _ptr(scales), M, _ptr(bias_bf16), _ptr(out), ldy, int(act), _stream()),
           "trdq_linear_act")
    return out


def trdq_linear_cfg(w: Weights, t: int, codes2, scales2, bias_bf16=None, out2=None):
    """Two row segments (conditional, unconditional) through one launch."""
    if out2 is None:
        done = (_native or _calls()).linear_cfg(w._h.value, w.N, t, codes2, scales2, bias_bf16)
        if done is not None:
            return _done(done, "trdq_linear_cfg")
    import torch
    Ms = [int(c.shape[0]) for c in codes2]
    empty = codes2[0].new_empty if type(codes2[0]) is torch.Tensor else _plain_empty(codes2[0])
    if out2 is None:
        out2 = [empty((m, w.N), dtype=torch.bfloat16) for m in Ms]
    vp2, i32_2, i64_2 = C.c_void_p * 2, C.c_int32 * 2, C.c_int64 * 2
    _check(lib().trdq_linear_cfg(w._h, int(t), vp2(*[_ptr(c) for c in codes2]), vp2(*[_ptr(s) for s in scales2]),
                                 i32_2(*Ms), _ptr(bias_bf16), vp2(*[_ptr(o) for o in out2]),
                                 i64_2(*[int(o.stride(0)) if m > 1 else w.N for o, m in zip(out2, Ms)]), _stream()),
           "trdq_linear_cfg")
    return out2


def trdq_linear_splitk_workspace(w: Weights, M: int) -> Tuple[int, int]:
    """(number of k ranges, workspace bytes) the split-K call would use for M rows."""
    splits, nbytes = C.c_int32(0), C.c_uint64(0)
    _check(lib().trdq_linear_splitk_workspace(w._h, int(M), C.byref(splits), C.byref(nbytes)), "trdq_linear_splitk_workspace")
    return splits.value, nbytes.value


def trdq_linear_splitk(w: Weights, t: int, codes, scales, bias_bf16=None, out=None, workspace=None):
    """trdq_linear with the reduction split over several CTAs per tile; `workspace` is a device tensor of at least
    the size trdq_linear_splitk_workspace reports (allocated here when omitted)."""
    done = (_native or _calls()).linear_splitk(w._h.value, w.N, t, codes, scales, bias_bf16, out, workspace)
    if done is not None:
        return _done(done, "trdq_linear_splitk")
    import torch
    M = int(codes.shape[0])
    empty = codes.new_empty if type(codes) is torch.Tensor else _plain_empty(codes)
    if out is None:
        out = empty((M, w.N), dtype=torch.bfloat16)
    splits, nbytes = trdq_linear_splitk_workspace(w, M)
    if workspace is None and nbytes:
        workspace = empty((nbytes,), dtype=torch.uint8)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    ldy = int(out.stride(0)) if M > 1 else w.N
    _check(lib().trdq_linear_splitk(w._h, int(t), _ptr(codes), _ptr(scales), M, _ptr(bias_bf16), _ptr(out), ldy, _ptr(workspace),
                                    ws_bytes, _stream()), "trdq_linear_splitk")
    return out


STATIC_SCRATCH_ELEMS = 2 * 1024 * 1024


def trdq_linear_splitk_static(w: Weights, t: int, codes, scales, bias_bf16, out):
    """Split-K linear whose partial sums go to the library's built-in scratch array: the call allocates nothing,
    so `out` must be passed in.  For callers that cannot allocate device memory where they call this."""
    M = int(codes.shape[0])
    ldy = int(out.stride(0)) if M > 1 else w.N
    _check(lib().trdq_linear_splitk_static(w._h, int(t), _ptr(codes), _ptr(scales), M, _ptr(bias_bf16), _ptr(out), ldy, _stream()),
           "trdq_linear_splitk_static")
    return out


def trdq_rotate_quantize_asym(rot: Rotation, t: int, X_bf16):
    """Asymmetric per-token quantizer of Eq. 1-3: (codes uint8 [M,K], scales fp32 [M], zero points int32 [M])."""
    done = (_native or _calls()).rotate_quantize_asym(rot._h.value, rot.K, t, X_bf16)
    if done is not None:
        return _done(done, "trdq_rotate_quantize_asym")
    import torch
    M = int(X_bf16.shape[0])
    empty = X_bf16.new_empty if type(X_bf16) is torch.Tensor else _plain_empty(X_bf16)
    codes = empty((M, rot.K), dtype=torch.uint8)
    scales = empty((M,), dtype=torch.float32)
    zp = empty((M,), dtype=torch.int32)
    ldx = int(X_bf16.stride(0)) if M > 1 else rot.K
    _check(lib().trdq_rotate_quantize_asym(rot._h, int(t), _ptr(X_bf16), ldx, M, _ptr(codes), _ptr(scales), _ptr(zp), _stream()),
           "trdq_rotate_quantize_asym")
    return codes, scales, zp


def trdq_linear_asym(w: Weights, t: int, codes, scales, zero_points, bias_bf16=None, out=None):
    done = (_native or _calls()).linear_asym(w._h.value, w.N, t, codes, scales, zero_points, bias_bf16, out)
    if done is not None:
        return _done(done, "trdq_linear_asym")
    import torch
    M = int(codes.shape[0])
    empty = codes.new_empty if type(codes) is torch.Tensor else _plain_empty(codes)
    if out is None:
        out = empty((M, w.N), dtype=torch.bfloat16)
    ldy = int(out.stride(0)) if M > 1 else w.N
    _check(lib().trdq_linear_asym(w._h, int(t), _ptr(codes), _ptr(scales), _ptr(zero_points), M, _ptr(bias_bf16), _ptr(out), ldy,
                                  _stream()), "trdq_linear_asym")
    return out


def trdq_gemm_i32(w: Weights, t: int, codes, out=None):
    """Raw int32 accumulators [M,N] of the integer GEMM (8-bit weights only)."""
    import torch
    M = int(codes.shape[0])
    empty = codes.new_empty if type(codes) is torch.Tensor else _plain_empty(codes)
    if out is None:
        out = empty((M, w.N), dtype=torch.int32)
    ld = int(out.stride(0)) if M > 1 else w.N
    _check(lib().trdq_gemm_i32(w._h, int(t), _ptr(codes), M, _ptr(out), ld, _stream()), "trdq_gemm_i32")
    return out


# ---- 8-bit floats with a scale for each block of 128 ----
def _here(where: str, *tensors) -> None:
    """These calls keep no object that would know its device: their tensors have to be on the current one."""
    import torch
    for x in tensors:
        if x is not None and (not x.is_cuda or x.device.index != torch.cuda.current_device()):
            raise TrdqError(10, f"{where} (a tensor is not on the current device)")


def _expect(where: str, x, shape, *dtypes) -> None:
    """x has this shape and one of these types, its last dimension side by side."""
    if x is None:
        return
    assert x.dtype in dtypes, f"{where}: {x.dtype} where {dtypes} is expected"
    if tuple(x.shape) != tuple(shape):
        raise TrdqError(2, f"{where} (shape {tuple(x.shape)} where {tuple(shape)} is expected)")
    assert x.numel() == 0 or x.stride(-1) == 1 or x.shape[-1] == 1, f"{where}: elements of a row do not lie side by side"


def _whole(where: str, *tensors) -> None:
    assert all(x is None or x.is_contiguous() for x in tensors), f"{where}: a tensor that has to be contiguous is not"


def _ld(x) -> int:
    return int(x.stride(0)) if x.shape[0] > 1 else int(x.shape[1])


def _rotation(rot: Optional[Rotation], where: str) -> Optional[int]:
    """Handle of a rotation, None for none.  A closed one is an error: its null handle would mean no rotation."""
    if rot is None:
        return None
    if not rot._h:
        raise TrdqError(1, f"{where} (the rotation is closed)")
    return rot._h.value


def _fp8_types():
    import torch
    return torch.float8_e4m3fn, torch.uint8


def trdq_fp8_quantize(X_bf16, rot: Optional[Rotation] = None, t: int = 0, codes=None, scales=None):
    """(codes e4m3 [M,K], scales fp32 [K/128,M]) of the rows of X, rotated by `rot` at time-step t if it is given."""
    where = "trdq_fp8_quantize"
    done = (_native or _calls()).fp8_quantize(_rotation(rot, where), t, X_bf16, codes, scales, 0)
    if done is not None:
        return _done(done, where)
    import torch
    assert X_bf16.dim() == 2 and X_bf16.dtype == torch.bfloat16
    M, K = int(X_bf16.shape[0]), int(X_bf16.shape[1])
    _here(where, X_bf16, codes, scales)
    _expect(where, X_bf16, (M, K), torch.bfloat16)
    if codes is None:
        codes = torch.empty((M, K), dtype=torch.float8_e4m3fn, device=X_bf16.device)
    if scales is None:
        scales = torch.empty((K // 128, M), dtype=torch.float32, device=X_bf16.device)
    _expect(where, codes, (M, K), *_fp8_types())
    _expect(where, scales, (K // 128, M), torch.float32)
    _whole(where, codes, scales)
    _check(lib().trdq_fp8_quantize(_rotation(rot, where), int(t), _ptr(X_bf16), _ld(X_bf16), M, K, _ptr(codes), _ptr(scales), _stream()), where)
    return codes, scales


def trdq_fp8_quantize_weights(W_bf16, rot: Optional[Rotation] = None, t: int = 0, codes=None, scales=None):
    """(codes e4m3 [N,K], scales fp32 [ceil(N/128),K/128]) of a weight matrix, for the group of time-step t if `rot` is given."""
    where = "trdq_fp8_quantize_weights"
    done = (_native or _calls()).fp8_quantize(_rotation(rot, where), t, W_bf16, codes, scales, 1)
    if done is not None:
        return _done(done, where)
    import torch
    assert W_bf16.dim() == 2 and W_bf16.dtype == torch.bfloat16
    N, K = int(W_bf16.shape[0]), int(W_bf16.shape[1])
    _here(where, W_bf16, codes, scales)
    if codes is None:
        codes = torch.empty((N, K), dtype=torch.float8_e4m3fn, device=W_bf16.device)
    if scales is None:
        scales = torch.empty(((N + 127) // 128, K // 128), dtype=torch.float32, device=W_bf16.device)
    _expect(where, codes, (N, K), *_fp8_types())
    _expect(where, scales, ((N + 127) // 128, K // 128), torch.float32)
    _whole(where, W_bf16, codes, scales)
    _check(lib().trdq_fp8_quantize_weights(_rotation(rot, where), int(t), _ptr(W_bf16), N, K, _ptr(codes), _ptr(scales), _stream()), where)
    return codes, scales


def trdq_fp8_linear(codes, scales, w_codes, w_scales, bias_bf16=None, out=None, act: int = ACT_NONE):
    """bf16 [M,N] product of block-scaled codes, with bias and activation."""
    where = "trdq_fp8_linear"
    done = (_native or _calls()).fp8_linear(codes, scales, w_codes, w_scales, bias_bf16, out, act)
    if done is not None:
        return _done(done, where)
    import torch
    assert codes.dim() == 2 and w_codes.dim() == 2
    M, K, N = int(codes.shape[0]), int(codes.shape[1]), int(w_codes.shape[0])
    _here(where, codes, scales, w_codes, w_scales, bias_bf16, out)
    if out is None:
        out = torch.empty((M, N), dtype=torch.bfloat16, device=codes.device)
    _expect(where, codes, (M, K), *_fp8_types())
    _expect(where, scales, (K // 128, M), torch.float32)
    _expect(where, w_codes, (N, K), *_fp8_types())
    _expect(where, w_scales, ((N + 127) // 128, K // 128), torch.float32)
    _expect(where, bias_bf16, (N,), torch.bfloat16)
    _expect(where, out, (M, N), torch.bfloat16)
    _whole(where, codes, scales, w_codes, w_scales, bias_bf16)
    _check(lib().trdq_fp8_linear(_ptr(codes), _ptr(scales), M, K, _ptr(w_codes), _ptr(w_scales), N, _ptr(bias_bf16), _ptr(out), _ld(out), int(act),
                                 _stream()), where)
    return out


# ---- norms before and after a block, with its gate and residual scale ----
NORM_NONE, NORM_LAYER, NORM_RMS = 0, 1, 2


def _gated_norm_op(where, X, branch, gate, shift, scale, weight, post_weight, norm, post_norm, rows_per_sample, eps, res_scale) -> GatedNormOp:
    import torch
    assert X.dim() == 2 and X.dtype in (torch.bfloat16, torch.float32)
    M, D = int(X.shape[0]), int(X.shape[1])
    rows = max(M, 1) if rows_per_sample is None else int(rows_per_sample)
    if rows < 1:
        raise TrdqError(2, f"{where} (rows_per_sample)")
    samples = (M + rows - 1) // rows
    _here(where, X, branch, gate, shift, scale, weight, post_weight)
    _expect(where, X, (M, D), X.dtype)
    _expect(where, branch, (M, D), torch.bfloat16)
    for p in (gate, shift, scale):
        _expect(where, p, (samples, D), torch.bfloat16)
    for p in (weight, post_weight):
        _expect(where, p, (D,), torch.bfloat16)

    def ld(p):
        return 0 if p is None else _ld(p)

    return GatedNormOp(M, D, rows, int(norm), int(post_norm), int(X.dtype == torch.float32), float(eps), float(res_scale), _ptr(X), _ld(X), _ptr(branch),
                       ld(branch), _ptr(gate), ld(gate), _ptr(shift), ld(shift), _ptr(scale), ld(scale), _ptr(weight), _ptr(post_weight))


def trdq_gated_norm(X, branch_bf16=None, gate=None, shift=None, scale=None, weight=None, post_weight=None, norm: int = NORM_LAYER,
                    post_norm: int = NORM_NONE, rows_per_sample: Optional[int] = None, eps: float = 1e-6, res_scale: float = 1.0, resid=None, out=None):
    """(R, H): R = res_scale * X + gate o post_norm(branch) o post_weight in X's type (`resid`: where to, X itself if wanted), and the bf16
    H = norm(R) o weight o (1 + scale) + shift.  gate, shift, scale: bf16 [samples, D], columns of a wider buffer if wanted."""
    where = "trdq_gated_norm"
    done = (_native or _calls()).gated_norm(X, branch_bf16, gate, shift, scale, weight, post_weight, norm, post_norm, rows_per_sample, eps, res_scale,
                                            resid, out)
    if done is not None:
        return _done(done, where)
    import torch
    op = _gated_norm_op(where, X, branch_bf16, gate, shift, scale, weight, post_weight, norm, post_norm, rows_per_sample, eps, res_scale)
    _here(where, resid, out)
    if resid is None:
        resid = torch.empty((op.M, op.D), dtype=X.dtype, device=X.device)
    if out is None:
        out = torch.empty((op.M, op.D), dtype=torch.bfloat16, device=X.device)
    _expect(where, resid, (op.M, op.D), X.dtype)
    _expect(where, out, (op.M, op.D), torch.bfloat16)
    _check(lib().trdq_gated_norm(C.byref(op), _ptr(resid), _ld(resid), _ptr(out), _ld(out), _stream()), where)
    return resid, out


def trdq_gated_norm_fp8(rot: Optional[Rotation], t: int, X, branch_bf16=None, gate=None, shift=None, scale=None, weight=None, post_weight=None,
                        norm: int = NORM_LAYER, post_norm: int = NORM_NONE, rows_per_sample: Optional[int] = None, eps: float = 1e-6,
                        res_scale: float = 1.0, resid=None, codes=None, scales=None):
    """trdq_gated_norm with H rotated (by `rot`, if it is given) and quantized in place of written: (R, codes e4m3 [M,D], scales fp32 [D/128,M])."""
    where = "trdq_gated_norm_fp8"
    done = (_native or _calls()).gated_norm_fp8(X, branch_bf16, gate, shift, scale, weight, post_weight, norm, post_norm, rows_per_sample, eps, res_scale,
                                                _rotation(rot, where), t, resid, codes, scales)
    if done is not None:
        return _done(done, where)
    import torch
    op = _gated_norm_op(where, X, branch_bf16, gate, shift, scale, weight, post_weight, norm, post_norm, rows_per_sample, eps, res_scale)
    _here(where, resid, codes, scales)
    if resid is None:
        resid = torch.empty((op.M, op.D), dtype=X.dtype, device=X.device)
    if codes is None:
        codes = torch.empty((op.M, op.D), dtype=torch.float8_e4m3fn, device=X.device)
    if scales is None:
        scales = torch.empty((op.D // 128, op.M), dtype=torch.float32, device=X.device)
    _expect(where, resid, (op.M, op.D), X.dtype)
    _expect(where, codes, (op.M, op.D), *_fp8_types())
    _expect(where, scales, (op.D // 128, op.M), torch.float32)
    _whole(where, codes, scales)
    _check(lib().trdq_gated_norm_fp8(C.byref(op), _rotation(rot, where), int(t), _ptr(resid), _ld(resid), _ptr(codes), _ptr(scales), _stream()),
           where)
    return resid, codes, scales


def trdq_gated_norm_backward(R, branch_bf16, dH_bf16, dR=None, gate=None, shift=None, scale=None, weight=None, post_weight=None,
                             norm: int = NORM_LAYER, post_norm: int = NORM_NONE, rows_per_sample: Optional[int] = None, eps: float = 1e-6,
                             res_scale: float = 1.0, dX=None, dB=None, workspace=None) -> dict:
    """Gradients of trdq_gated_norm from the stored R, the gradient of H and (or None) what arrives at R from elsewhere: dx in R's type, db in bf16 and
    those of the parameters that are given in fp32, under the names dx, db, dgate, dshift, dscale, dweight, dpost_weight (None: no such input)."""
    where = "trdq_gated_norm_backward"
    names = ("dx", "db", "dgate", "dshift", "dscale", "dweight", "dpost_weight")
    if dX is None and dB is None and workspace is None:
        done = (_native or _calls()).gated_norm_backward(R, branch_bf16, gate, shift, scale, weight, post_weight, norm, post_norm, rows_per_sample, eps,
                                                         res_scale, dH_bf16, dR)
        if done is not None:
            return dict(zip(names, _done(done, where)))
    import torch
    op = _gated_norm_op(where, R, branch_bf16, gate, shift, scale, weight, post_weight, norm, post_norm, rows_per_sample, eps, res_scale)
    M, D, dev = op.M, op.D, R.device
    samples = (M + op.rows_per_sample - 1) // op.rows_per_sample
    _here(where, dH_bf16, dR, dX, dB, workspace)
    if dX is None:
        dX = torch.empty((M, D), dtype=R.dtype, device=dev)
    if dB is None and branch_bf16 is not None:
        dB = torch.empty((M, D), dtype=torch.bfloat16, device=dev)
    _expect(where, dH_bf16, (M, D), torch.bfloat16)
    _expect(where, dR, (M, D), R.dtype)
    _expect(where, dX, (M, D), R.dtype)
    _expect(where, dB, (M, D), torch.bfloat16)

    def grad(p, *shape):
        return None if p is None else torch.empty(shape, dtype=torch.float32, device=dev)

    dgate, dshift, dscale = grad(gate, samples, D), grad(shift, samples, D), grad(scale, samples, D)
    dweight, dpost_weight = grad(weight, D), grad(post_weight, D)
    if workspace is None and any(g is not None for g in (dgate, dshift, dscale, dweight, dpost_weight)):
        n = C.c_uint64(0)
        _check(lib().trdq_gated_norm_backward_workspace(C.byref(op), C.byref(n)), where)
        workspace = torch.empty((max(int(n.value), 16),), dtype=torch.uint8, device=dev)

    def ld(p):
        return 0 if p is None else _ld(p)

    _check(lib().trdq_gated_norm_backward(C.byref(op), _ptr(dH_bf16), ld(dH_bf16), _ptr(dR), ld(dR), _ptr(dX), ld(dX), _ptr(dB), ld(dB), _ptr(dgate),
                                          _ptr(dshift), _ptr(dscale), _ptr(dweight), _ptr(dpost_weight), _ptr(workspace),
                                          0 if workspace is None else workspace.numel() * workspace.element_size(), _stream()), where)
    return dict(zip(names, (dX, dB, dgate, dshift, dscale, dweight, dpost_weight)))


class LayerList:
    """A fixed list of trdq_layer_op records (one denoising step's quantized linears).  Holds
    references to every tensor and handle it points to."""

    def __init__(self):
        self._keep = []
        self._extra = []
        self._ops = []
        self._array = None

    def add(self, rot: Rotation, w: Weights, X_bf16, codes, scales, bias_bf16, Y_bf16, act: int = 0, workspace=None) -> None:
        M = int(X_bf16.shape[0])
        assert X_bf16.stride(1) == 1 and Y_bf16.stride(1) == 1 and codes.is_contiguous()
        self._ops.append(LayerOp(rot._h, w._h, _ptr(X_bf16), int(X_bf16.stride(0)) if M > 1 else rot.K, M, _ptr(codes),
                                 _ptr(scales), _ptr(bias_bf16), _ptr(Y_bf16), int(Y_bf16.stride(0)) if M > 1 else w.N, int(act),
                                 _ptr(workspace), 0 if workspace is None else int(workspace.numel() * workspace.element_size())))
        self._keep.append((rot, w, X_bf16, codes, scales, bias_bf16, Y_bf16))
        self._extra.append(workspace)
        self._array = None

    def __len__(self) -> int:
        return len(self._ops)

    def array(self):
        if self._array is None:
            self._array = (LayerOp * len(self._ops))(*self._ops)
        return self._array


def trdq_run_layers(layers: LayerList, t: int, first: int = 0, count: Optional[int] = None) -> None:
    """All (or a slice of) the layer ops at time-step t on the current stream."""
    n = len(layers) - first if count is None else count
    arr = layers.array()
    ptr = C.cast(C.byref(arr, first * C.sizeof(LayerOp)), C.POINTER(LayerOp))
    _check(lib().trdq_run_layers(ptr, int(n), int(t), _stream()), "trdq_run_layers")


def trdq_kernel_choice(stage: int, M: int, K: int, N: int = 0, wbits: int = 8) -> str:
    """Name of the kernel trdq_rotate_quantize (stage 0), trdq_linear (stage 1) or trdq_fp8_linear (stage 2) runs for this shape on the current device."""
    buf = C.create_string_buffer(96)
    _check(lib().trdq_kernel_choice(int(stage), int(M), int(K), int(N), int(wbits), buf, 96), "trdq_kernel_choice")
    return buf.value.decode()


def trdq_measure_mma_ceiling(mmas_per_cluster: int) -> int:
    """Launches the tensor-pipe-only kernel on the current stream; returns the integer operations the launch performs."""
    clusters = C.c_int32(0)
    _check(lib().trdq_measure_mma_ceiling(int(mmas_per_cluster), C.byref(clusters), _stream()), "trdq_measure_mma_ceiling")
    return clusters.value * int(mmas_per_cluster) * 2 * 256 * 256 * 32


def trdq_selftest_wait_expiry() -> None:
    """Launches the kernel whose only barrier is never signalled (its wait expires after 20 ms)."""
    _check(lib().trdq_selftest_wait_expiry(_stream()), "trdq_selftest_wait_expiry")


def trdq_selftest_fp8_linear_expiry(codes, scales, w_codes, w_scales) -> None:
    """Launches the block-scaled product's kernel of CTA pairs without the copies of its operands (its waits expire after a second)."""
    import torch
    M, K, N = int(codes.shape[0]), int(codes.shape[1]), int(w_codes.shape[0])
    where = "trdq_selftest_fp8_linear_expiry"
    _here(where, codes, scales, w_codes, w_scales)
    _expect(where, codes, (M, K), *_fp8_types())
    _expect(where, scales, (K // 128, M), torch.float32)
    _expect(where, w_codes, (N, K), *_fp8_types())
    _expect(where, w_scales, ((N + 127) // 128, K // 128), torch.float32)
    _whole(where, codes, scales, w_codes, w_scales)
    out = torch.empty((M, N), dtype=torch.bfloat16, device=codes.device)
    _check(lib().trdq_selftest_fp8_linear_expiry(_ptr(codes), _ptr(scales), M, K, _ptr(w_codes), _ptr(w_scales), N, _ptr(out), N, _stream()), where)


def trdq_device_status() -> int:
    """Synchronises; returns the raw status word (0 = no bounded wait expired) and clears it."""
    word = C.c_uint32(0)
    st = lib().trdq_device_status(C.byref(word))
    if st not in (0, 9):
        raise TrdqError(st, "trdq_device_status")
    return word.value
