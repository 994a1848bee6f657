"""Thin ctypes binding of the C ABI declared in ``include/dvdq.h``.

Argument marshalling only: every function takes torch CUDA tensors (device memory) and a
stream, checks dtypes, passes raw pointers and raises :class:`DvdqError` on a non-zero
status.  No step of the path runs in Python or on the CPU, and there is no fallback: if the
CUDA library is missing, importing the functions fails loudly.
"""
from __future__ import annotations

import ctypes as C
import os
import struct
from typing import Optional

import torch

from . import build as _build

# status codes of include/dvdq.h
OK, ERR_NULL, ERR_SHAPE, ERR_BITS, ERR_ROT_BLOCK, ERR_ALIGN, ERR_WORKSPACE, ERR_BLOB, ERR_ARCH, \
    ERR_CUDA, ERR_DEVICE_TIMEOUT, ERR_UNSUPPORTED = range(12)

EXPORTS = [
    "dvdq_status_string", "dvdq_version", "dvdq_act_codes_bytes", "dvdq_act_codes_bytes_q", "dvdq_act_scales_count", "dvdq_weight_blob_bytes",
    "dvdq_qlinear_workspace_bytes", "dvdq_rotate_quantize", "dvdq_pack_weights", "dvdq_qgemm",
    "dvdq_qlinear", "dvdq_qlinear_static", "dvdq_qgemm_fused_rq", "dvdq_qgemm_int32", "dvdq_pack_act_codes", "dvdq_unpack_act_codes",
    "dvdq_unpack_weights", "dvdq_last_device_status",
    "dvdq_rotate_weights", "dvdq_quantize_weights_symmetric", "dvdq_int8_mma_ceiling", "dvdq_debug_wait_timeout",
    "dvdq_weight_operand_bytes", "dvdq_widen_weights",
    "dvdq_bgr_quantize", "dvdq_gbs_l1_terms", "dvdq_gbs_init", "dvdq_gbs_next_bits", "dvdq_gbs_observe",
    "dvdq_linear_workspace_bytes", "dvdq_linear", "dvdq_linear_backward_workspace_bytes", "dvdq_linear_backward",
    "dvdq_rope_frequencies", "dvdq_rope_table", "dvdq_rope",
    "dvdq_group_norm_workspace_bytes", "dvdq_group_norm", "dvdq_group_norm_backward",
    "dvdq_rms_norm", "dvdq_rms_norm_backward_workspace_bytes", "dvdq_rms_norm_backward", "dvdq_quantize_rows",
    "dvdq_linear_int8_workspace_bytes", "dvdq_linear_int8",
]

# element types, activations and rotary options of include/dvdq.h
BF16, F16, F32 = range(3)
ACT_NONE, ACT_GELU_TANH, ACT_SILU = range(3)
ROPE_PAIRS, ROPE_HALVES = range(2)
ROPE_PLAIN, ROPE_LINEAR, ROPE_BASE, ROPE_BY_PARTS = range(4)
_DTYPES = {torch.bfloat16: BF16, torch.float16: F16, torch.float32: F32}


class DvdqError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: status {status} ({status_string(status)})")


class ActQuant(C.Structure):
    """dvdq_act_quant: the activation quantizer of Eq. 10 (bits, rotation block, scale granularity)
    and how its codes are stored (container_bits: 0 = packed, 8 = one int8 per code)."""
    _fields_ = [("bits", C.c_int32), ("rot_block", C.c_int32), ("scale_group", C.c_int32),
                ("container_bits", C.c_int32)]


class Weights(C.Structure):
    """dvdq_weights: host handle of a packed weight blob."""
    _fields_ = [("magic", C.c_uint32), ("version", C.c_uint32), ("N", C.c_int64), ("K", C.c_int64),
                ("rot_block", C.c_int32), ("k_layout", C.c_int32), ("blob", C.c_void_p),
                ("blob_bytes", C.c_uint64), ("operand", C.c_void_p), ("operand_bytes", C.c_uint64)]


class RopeTensor(C.Structure):
    """dvdq_rope_tensor: one of q and k, [B, S, heads, head_dim], strides in elements."""
    _fields_ = [("x", C.c_void_p), ("y", C.c_void_p), ("heads", C.c_int64),
                ("x_batch", C.c_int64), ("x_token", C.c_int64), ("x_head", C.c_int64),
                ("y_batch", C.c_int64), ("y_token", C.c_int64), ("y_head", C.c_int64)]


class GbsState(C.Structure):
    """dvdq_gbs_state: host-side state of the delta-guided bit switching (Sec. 3.3)."""
    _fields_ = [("delta", C.c_double), ("b_low", C.c_int32), ("b_high", C.c_int32), ("accumulated", C.c_double),
                ("steps", C.c_int64), ("high_steps", C.c_int64)]


_lib = None


def lib_path() -> str:
    return _build.LIB_PATH


def load():
    """dlopen the in-tree library (building it first if the sources are newer)."""
    global _lib
    if _lib is not None:
        return _lib
    path = _build.LIB_PATH
    if _build.is_stale():
        try:
            path = _build.build_library()
        except Exception as e:  # no nvcc on this machine and no prebuilt library
            if not os.path.exists(path):
                raise RuntimeError(f"CUDA library {path} is missing and cannot be built: {e}") from e
    lib = C.CDLL(path)
    i32, i64, p, sz = C.c_int32, C.c_int64, C.c_void_p, C.c_size_t
    aq, wp = C.POINTER(ActQuant), C.POINTER(Weights)
    sig = {
        "dvdq_status_string": (C.c_char_p, [C.c_int]),
        "dvdq_version": (i32, []),
        "dvdq_act_codes_bytes": (sz, [i64, i64, i32]),
        "dvdq_act_codes_bytes_q": (sz, [i64, i64, aq]),
        "dvdq_act_scales_count": (sz, [i64, i64, aq]),
        "dvdq_weight_blob_bytes": (sz, [i64, i64]),
        "dvdq_weight_operand_bytes": (sz, [i64, i64]),
        "dvdq_widen_weights": (C.c_int, [wp, p, sz, wp, p]),
        "dvdq_qlinear_workspace_bytes": (sz, [i64, i64, aq]),
        "dvdq_rotate_quantize": (C.c_int, [p, i64, i64, i64, aq, p, p, p, p]),
        "dvdq_pack_weights": (C.c_int, [p, p, p, i64, i64, i32, p, wp, p]),
        "dvdq_qgemm": (C.c_int, [p, p, p, i64, aq, wp, p, i32, p, i64, p]),
        "dvdq_qlinear": (C.c_int, [p, i64, i64, aq, wp, p, i32, p, i64, p, sz, p]),
        "dvdq_qlinear_static": (C.c_int, [p, i64, i64, aq, wp, p, i32, p, i64, p]),
        "dvdq_qgemm_int32": (C.c_int, [p, p, i64, aq, wp, p, i64, p]),
        "dvdq_qgemm_fused_rq": (C.c_int, [p, p, p, i64, aq, wp, p, i32, aq, p, p, p, p, i64, p]),
        "dvdq_pack_act_codes": (C.c_int, [p, i64, i64, aq, p, p, p]),
        "dvdq_unpack_act_codes": (C.c_int, [p, i64, i64, aq, p, p]),
        "dvdq_unpack_weights": (C.c_int, [wp, p, p, p, p]),
        "dvdq_last_device_status": (C.c_int, [C.POINTER(C.c_uint32)]),
        "dvdq_bgr_quantize": (C.c_int, [p, i64, i64, i32, C.c_double, i32, p, p, p, p]),
        "dvdq_rotate_weights": (C.c_int, [p, i64, i64, i64, i32, p, p]),
        "dvdq_quantize_weights_symmetric": (C.c_int, [p, i64, i64, i64, i32, p, wp, p]),
        "dvdq_int8_mma_ceiling": (C.c_int, [i32, C.POINTER(C.c_int64), p]),
        "dvdq_debug_wait_timeout": (C.c_int, [C.c_uint64, p]),
        "dvdq_gbs_l1_terms": (C.c_int, [p, p, i64, p, p]),
        "dvdq_gbs_init": (C.c_int, [C.POINTER(GbsState), C.c_double, i32, i32]),
        "dvdq_gbs_next_bits": (i32, [C.POINTER(GbsState)]),
        "dvdq_gbs_observe": (C.c_int, [C.POINTER(GbsState), C.c_double, C.c_double]),
        "dvdq_linear_workspace_bytes": (sz, [i64, i64, i64]),
        "dvdq_linear": (C.c_int, [p, i64, i64, p, i64, i64, i64, p, p, i64, i32, p, i64, p, i64, i32, p, sz, p]),
        "dvdq_linear_backward_workspace_bytes": (sz, [i64, i64, i64, i32]),
        "dvdq_linear_backward": (C.c_int, [p, i64, p, i64, p, i64, p, i64, i64, i64, i64, i32, p, i64, p, i64, p, i32, p, sz, p]),
        "dvdq_rope_frequencies": (C.c_int, [i32, C.c_double, i32, C.c_double, C.c_double, C.c_double, C.c_double,
                                            C.POINTER(C.c_double), C.POINTER(C.c_double)]),
        "dvdq_rope_table": (C.c_int, [C.POINTER(C.c_double), C.POINTER(i32), i32, p, i64, i32, C.c_double, p, p]),
        "dvdq_rope": (C.c_int, [C.POINTER(RopeTensor), C.POINTER(RopeTensor), i64, i64, i32, i32, p, i64, p, i64, i32, i32, i32, p]),
        "dvdq_group_norm_workspace_bytes": (sz, [i64, i64, i64, i64]),
        "dvdq_group_norm": (C.c_int, [p, i64, i64, i64, i64, i64, i64, p, p, i32, C.c_float, i32, p, i64, i64, p, p, i32, p, sz, p]),
        "dvdq_group_norm_backward": (C.c_int, [p, i64, i64, p, i64, i64, p, p, i64, i64, i64, i64, p, p, i32, i32, p, i64, i64, p, p,
                                               i32, p, sz, p]),
        "dvdq_rms_norm": (C.c_int, [C.c_char_p, p]),
        "dvdq_rms_norm_backward_workspace_bytes": (sz, [i64, i64, i64]),
        "dvdq_rms_norm_backward": (C.c_int, [C.c_char_p, p]),
        "dvdq_quantize_rows": (C.c_int, [p, i64, i64, i64, p, i64, p, i32, p]),
        "dvdq_linear_int8_workspace_bytes": (sz, [i64, i64, i64]),
        "dvdq_linear_int8": (C.c_int, [C.c_char_p, p]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    _lib = lib
    return lib


def status_string(status: int) -> str:
    return load().dvdq_status_string(int(status)).decode()


def _check(status: int, where: str):
    if status != OK:
        raise DvdqError(status, where)


def _ptr(t: Optional[torch.Tensor], dtype=None, name="tensor"):
    if t is None:
        return None
    if not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    return C.c_void_p(t.data_ptr())


def _stream(stream) -> C.c_void_p:
    if stream is None:
        stream = torch.cuda.current_stream()
    return C.c_void_p(stream.cuda_stream)


def _row_major(t: torch.Tensor, name: str) -> int:
    if t.dim() != 2 or t.stride(1) != 1:
        raise TypeError(f"{name} must be 2-D with unit inner stride")
    return t.stride(0)


# ------------------------------------------------------------------ size queries

def dvdq_version() -> int:
    return int(load().dvdq_version())


def dvdq_act_codes_bytes(M: int, K: int, bits: int) -> int:
    return int(load().dvdq_act_codes_bytes(M, K, bits))


def dvdq_act_codes_bytes_q(M: int, K: int, q: ActQuant) -> int:
    return int(load().dvdq_act_codes_bytes_q(M, K, C.byref(q)))


def dvdq_act_scales_count(M: int, K: int, q: ActQuant) -> int:
    return int(load().dvdq_act_scales_count(M, K, C.byref(q)))


def dvdq_weight_blob_bytes(N: int, K: int) -> int:
    return int(load().dvdq_weight_blob_bytes(N, K))


def dvdq_qlinear_workspace_bytes(M: int, K: int, q: ActQuant) -> int:
    return int(load().dvdq_qlinear_workspace_bytes(M, K, C.byref(q)))


# ------------------------------------------------------------------ the path

def dvdq_rotate_quantize(X: torch.Tensor, q: ActQuant, codes: torch.Tensor, scales: torch.Tensor,
                         code_sums: torch.Tensor, stream=None) -> None:
    ldx = _row_major(X, "X")
    M, K = X.shape
    _check(load().dvdq_rotate_quantize(_ptr(X, torch.bfloat16, "X"), M, K, ldx, C.byref(q),
                                       _ptr(codes, torch.uint8, "codes"), _ptr(scales, torch.float32, "scales"),
                                       _ptr(code_sums, torch.int32, "code_sums"), _stream(stream)),
           "dvdq_rotate_quantize")


def dvdq_pack_weights(Wq: torch.Tensor, delta: torch.Tensor, zero: torch.Tensor, rot_block: int,
                      blob: torch.Tensor, stream=None) -> Weights:
    N, K = Wq.shape
    if not Wq.is_contiguous():
        raise TypeError("Wq must be contiguous")
    w = Weights()
    _check(load().dvdq_pack_weights(_ptr(Wq, torch.uint8, "Wq"), _ptr(delta, torch.float32, "delta"),
                                    _ptr(zero, torch.int32, "zero"), N, K, rot_block,
                                    _ptr(blob, torch.uint8, "blob"), C.byref(w), _stream(stream)),
           "dvdq_pack_weights")
    return w


def dvdq_qgemm(codes: torch.Tensor, scales: torch.Tensor, code_sums: torch.Tensor, M: int, q: ActQuant,
               w: Weights, bias: Optional[torch.Tensor], act: int, Y: torch.Tensor, stream=None) -> None:
    ldy = _row_major(Y, "Y")
    _check(load().dvdq_qgemm(_ptr(codes, torch.uint8, "codes"), _ptr(scales, torch.float32, "scales"),
                             _ptr(code_sums, torch.int32, "code_sums"), M, C.byref(q), C.byref(w),
                             _ptr(bias, torch.bfloat16, "bias"), act, _ptr(Y, torch.bfloat16, "Y"), ldy,
                             _stream(stream)), "dvdq_qgemm")


def dvdq_qgemm_fused_rq(codes: torch.Tensor, scales: torch.Tensor, code_sums: torch.Tensor, M: int, q: ActQuant,
                        w: Weights, bias: Optional[torch.Tensor], act: int, q_next: ActQuant, codes_next: torch.Tensor,
                        scales_next: torch.Tensor, code_sums_next: torch.Tensor, Y: Optional[torch.Tensor] = None,
                        stream=None) -> None:
    """dvdq_qgemm whose epilogue writes the next layer's codes / scales / code sums
    (rot_block = scale_group = 256, one int8 per code) instead of bf16; Y, if given, also gets the bf16 output."""
    ldy = _row_major(Y, "Y") if Y is not None else 0
    _check(load().dvdq_qgemm_fused_rq(_ptr(codes, torch.uint8, "codes"), _ptr(scales, torch.float32, "scales"),
                                      _ptr(code_sums, torch.int32, "code_sums"), M, C.byref(q), C.byref(w),
                                      _ptr(bias, torch.bfloat16, "bias"), act, C.byref(q_next),
                                      _ptr(codes_next, torch.uint8, "codes_next"), _ptr(scales_next, torch.float32, "scales_next"),
                                      _ptr(code_sums_next, torch.int32, "code_sums_next"), _ptr(Y, torch.bfloat16, "Y"), ldy,
                                      _stream(stream)), "dvdq_qgemm_fused_rq")


def dvdq_qlinear(X: torch.Tensor, q: ActQuant, w: Weights, bias: Optional[torch.Tensor], act: int,
                 Y: torch.Tensor, workspace: torch.Tensor, stream=None) -> None:
    ldx = _row_major(X, "X")
    ldy = _row_major(Y, "Y")
    M = X.shape[0]
    _check(load().dvdq_qlinear(_ptr(X, torch.bfloat16, "X"), M, ldx, C.byref(q), C.byref(w),
                               _ptr(bias, torch.bfloat16, "bias"), act, _ptr(Y, torch.bfloat16, "Y"), ldy,
                               _ptr(workspace, torch.uint8, "workspace"), workspace.numel(), _stream(stream)),
           "dvdq_qlinear")


STATIC_SCRATCH_BYTES = 16 * 1024 * 1024


def dvdq_qlinear_static(X: torch.Tensor, q: ActQuant, w: Weights, bias: Optional[torch.Tensor], act: int,
                        Y: torch.Tensor, stream=None) -> None:
    """dvdq_qlinear for callers that cannot allocate: the intermediate codes live in a fixed
    STATIC_SCRATCH_BYTES array inside the library (shared by all calls on a device, so calls
    must not overlap; larger problems are refused with ERR_WORKSPACE)."""
    ldx = _row_major(X, "X")
    ldy = _row_major(Y, "Y")
    _check(load().dvdq_qlinear_static(_ptr(X, torch.bfloat16, "X"), X.shape[0], ldx, C.byref(q), C.byref(w),
                                      _ptr(bias, torch.bfloat16, "bias"), act, _ptr(Y, torch.bfloat16, "Y"), ldy,
                                      _stream(stream)), "dvdq_qlinear_static")


# ------------------------------------------------------------------ around the quantized layers

def _address(t: Optional[torch.Tensor], dtype, name: str) -> Optional[int]:
    """Device address of a tensor whose dtype is as required; None for None."""
    if t is None:
        return None
    if not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor")
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    return t.data_ptr()


def _vector(t: Optional[torch.Tensor], dtype, n: int, name: str) -> Optional[int]:
    if t is None:
        return None
    if t.dim() != 1 or len(t) != n or (n > 1 and t.stride(0) != 1):
        raise TypeError(f"{name} must be a dense vector of {n} values")
    return _address(t, dtype, name)


def _matrix(t: Optional[torch.Tensor], dtype, rows: int, cols: int, name: str):
    """(address, row pitch) of a [rows, cols] matrix with unit inner stride."""
    if t is None:
        return None, 0
    shape = t.shape
    if len(shape) != 2 or shape[0] != rows or shape[1] != cols:
        raise TypeError(f"{name} must have shape {(rows, cols)}, got {tuple(shape)}")
    pitch, inner = t.stride()
    if cols > 1 and inner != 1:
        raise TypeError(f"{name} must have unit inner stride")
    return _address(t, dtype, name), pitch


_ANY_FLOAT, _HALF_FLOAT = (BF16, F16, F32), (BF16, F16)


def _element_type(t: torch.Tensor, name: str, allowed) -> int:
    code = _DTYPES.get(t.dtype, -1)
    if code not in allowed:
        raise TypeError(f"{name} must be one of {[str(k) for k, v in _DTYPES.items() if v in allowed]}, got {t.dtype}")
    return code


def _room(workspace: Optional[torch.Tensor]):
    if workspace is None:
        return None, 0
    return _address(workspace, torch.uint8, "workspace"), workspace.numel()


def _raw_stream(stream, t: torch.Tensor) -> int:
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(t.device.index)
    return stream.cuda_stream


def dvdq_linear_workspace_bytes(M: int, N: int, K: int) -> int:
    return int(load().dvdq_linear_workspace_bytes(M, N, K))


def dvdq_linear(X: torch.Tensor, W: torch.Tensor, bias: Optional[torch.Tensor], residual: Optional[torch.Tensor], act: int,
                Y: torch.Tensor, Z: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """Y = act(X W^T + bias) + residual for X [M, K], W [N, K] in bf16 or fp16; Z, if given, receives the
    pre-activation for dvdq_linear_backward.  residual may be Y itself.  Rows start on 16 bytes (pitches
    are multiples of 8 elements); workspace: dvdq_linear_workspace_bytes(M, N, K) bytes, None where that is 0."""
    dt = X.dtype
    code = _element_type(X, "X", _HALF_FLOAT)
    if X.dim() != 2 or W.dim() != 2:
        raise TypeError("X and W must be 2-D")
    (M, K), N = X.shape, W.shape[0]
    x, ldx = _matrix(X, dt, M, K, "X")
    w, ldw = _matrix(W, dt, N, K, "W")
    r, ldr = _matrix(residual, dt, M, N, "residual")
    y, ldy = _matrix(Y, dt, M, N, "Y")
    z, ldz = _matrix(Z, dt, M, N, "Z")
    ws, room = _room(workspace)
    _check(load().dvdq_linear(x, M, ldx, w, N, K, ldw, _vector(bias, dt, N, "bias"), r, ldr, act, y, ldy, z, ldz, code, ws, room,
                              _raw_stream(stream, X)), "dvdq_linear")


def dvdq_linear_backward_workspace_bytes(M: int, N: int, K: int, act: int) -> int:
    return int(load().dvdq_linear_backward_workspace_bytes(M, N, K, act))


def dvdq_linear_backward(dY: torch.Tensor, Z: Optional[torch.Tensor], X: Optional[torch.Tensor], W: Optional[torch.Tensor], act: int,
                         dX: Optional[torch.Tensor], dW: Optional[torch.Tensor], dbias: Optional[torch.Tensor],
                         workspace: torch.Tensor, stream=None) -> None:
    """Gradients of dvdq_linear: dX [M, K], dW [N, K] (dY's type), dbias fp32 [N], each written if given.  Z is
    the pre-activation (not read without an activation); X is needed for dW, W for dX.  The residual's gradient is dY."""
    dt = dY.dtype
    code = _element_type(dY, "dY", _HALF_FLOAT)
    if dY.dim() != 2:
        raise TypeError("dY must be 2-D")
    M, N = dY.shape
    given = next((t for t in (X, W, dX, dW) if t is not None), None)
    K = given.shape[1] if given is not None and given.dim() == 2 else 8  # only dbias asked for: no K is read
    dy, lddy = _matrix(dY, dt, M, N, "dY")
    z, ldz = _matrix(Z, dt, M, N, "Z")
    x, ldx = _matrix(X, dt, M, K, "X")
    w, ldw = _matrix(W, dt, N, K, "W")
    dx, lddx = _matrix(dX, dt, M, K, "dX")
    dw, lddw = _matrix(dW, dt, N, K, "dW")
    ws, room = _room(workspace)
    _check(load().dvdq_linear_backward(dy, lddy, z, ldz, x, ldx, w, ldw, M, N, K, act, dx, lddx, dw, lddw,
                                       _vector(dbias, torch.float32, N, "dbias"), code, ws, room, _raw_stream(stream, dY)),
           "dvdq_linear_backward")


def dvdq_rope_frequencies(rot_dim: int, theta: float = 10000.0, scaling: int = ROPE_PLAIN, factor: float = 1.0,
                          original_length: float = 0.0, beta_fast: float = 32.0, beta_slow: float = 1.0):
    """(list of rot_dim / 2 frequencies, amplitude) on the host, optionally stretched for long contexts."""
    freqs, amplitude = (C.c_double * max(1, rot_dim // 2))(), C.c_double(0.0)
    _check(load().dvdq_rope_frequencies(rot_dim, theta, scaling, factor, original_length, beta_fast, beta_slow, freqs,
                                        C.byref(amplitude)), "dvdq_rope_frequencies")
    return list(freqs), amplitude.value


def dvdq_rope_table(freqs, positions: Optional[torch.Tensor], table: torch.Tensor, axis_of_pair=None, amplitude: float = 1.0,
                    stream=None) -> None:
    """table [rows, pairs, 2] fp32 = amplitude * (cos, sin)(position * frequency).  positions: int32 [rows] or
    [rows, axes], or None (position = row); axis_of_pair: for each pair, which axis it turns with."""
    pairs = len(freqs)
    if table.dim() != 3 or table.shape[1:] != (pairs, 2) or not table.is_contiguous():
        raise TypeError(f"table must be dense [rows, {pairs}, 2]")
    rows, axes = table.shape[0], 1
    if positions is not None:
        axes = 1 if positions.dim() == 1 else positions.shape[-1]
        if positions.dim() not in (1, 2) or positions.shape[0] != rows or not positions.is_contiguous():
            raise TypeError("positions must be dense [rows] or [rows, axes]")
    if axis_of_pair is not None and len(axis_of_pair) != pairs:
        raise TypeError("axis_of_pair must name an axis for each pair")
    axis = (C.c_int32 * pairs)(*axis_of_pair) if axis_of_pair is not None else None
    _check(load().dvdq_rope_table((C.c_double * pairs)(*freqs), axis, pairs, _address(positions, torch.int32, "positions"), rows, axes,
                                  amplitude, _address(table, torch.float32, "table"), _raw_stream(stream, table)), "dvdq_rope_table")


def _rope_tensor(x: torch.Tensor, y: torch.Tensor, B: int, S: int, D: int, dtype, name: str) -> RopeTensor:
    shape = x.shape
    if len(shape) != 4 or shape[0] != B or shape[1] != S or shape[3] != D:
        raise TypeError(f"{name} must be [B, S, heads, head_dim] like q")
    if y.shape != shape:
        raise TypeError(f"{name}_out must have shape {tuple(shape)}, got {tuple(y.shape)}")
    xb, xs, xh, xd = x.stride()
    yb, ys, yh, yd = y.stride()
    if D > 1 and (xd != 1 or yd != 1):
        raise TypeError(f"{name} must have unit stride inside a head")
    return RopeTensor(_address(x, dtype, name), _address(y, dtype, name + "_out"), shape[2], xb, xs, xh, yb, ys, yh)


def dvdq_rope(q: torch.Tensor, k: Optional[torch.Tensor], table: torch.Tensor, rows: Optional[torch.Tensor], layout: int,
              inverse: bool, q_out: torch.Tensor, k_out: Optional[torch.Tensor] = None, stream=None) -> None:
    """Rotates q [B, S, Hq, D] and k [B, S, Hk, D] (any strides with unit stride inside a head) into q_out and k_out, which
    may be q and k themselves.  table [rows, rot_dim / 2, 2] of dvdq_rope_table; rows: int32 [B, S] or [S], the table
    row of each token (None: token s takes row s).  inverse=True: the gradient."""
    dt = q.dtype
    code = _element_type(q, "q", _ANY_FLOAT)
    if q.dim() != 4:
        raise TypeError("q must be [B, S, heads, head_dim]")
    B, S, _, D = q.shape
    if (k is None) != (k_out is None):
        raise TypeError("k and k_out come together")
    table_rows, pairs, two = table.shape if table.dim() == 3 else (0, 0, 0)
    if two != 2 or not table.is_contiguous():
        raise TypeError("table must be dense [rows, rot_dim / 2, 2]")
    batch, index = 0, None
    if rows is not None:
        shape, strides = rows.shape, rows.stride()
        if shape != (B, S) and shape != (S,):
            raise TypeError("rows must be [B, S] or [S]")
        if S > 1 and strides[-1] != 1:
            raise TypeError("rows must have unit stride along the tokens")
        batch = strides[0] if len(shape) == 2 else 0
        index = _address(rows, torch.int32, "rows")
    _check(load().dvdq_rope(_rope_tensor(q, q_out, B, S, D, dt, "q"), None if k is None else _rope_tensor(k, k_out, B, S, D, dt, "k"),
                            B, S, D, 2 * pairs, _address(table, torch.float32, "table"), table_rows, index, batch, layout,
                            1 if inverse else 0, code, _raw_stream(stream, q)), "dvdq_rope")


def dvdq_group_norm_workspace_bytes(N: int, S: int, C_: int, G: int) -> int:
    return int(load().dvdq_group_norm_workspace_bytes(N, S, C_, G))


def _places(t: Optional[torch.Tensor], dtype, shape, name: str):
    """(address, sample pitch, place pitch) of an [N, S, C] tensor with unit stride of channels."""
    if t is None:
        return None, 0, 0
    if t.shape != shape:
        raise TypeError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    st = t.stride()
    if shape[2] > 1 and st[2] != 1:
        raise TypeError(f"{name} must have unit stride of channels (channels last)")
    return _address(t, dtype, name), st[0], st[1]


def _norm_params(gamma, beta, dt, code: int, channels: int):
    given = gamma if gamma is not None else beta
    pt = dt if given is None else given.dtype
    if pt is not dt and pt is not torch.float32:
        raise TypeError(f"gamma and beta must be {dt} or torch.float32, got {pt}")
    return _vector(gamma, pt, channels, "gamma"), _vector(beta, pt, channels, "beta"), code if pt is dt else F32


def _group_stats(t: Optional[torch.Tensor], N: int, G: int, name: str):
    if t is not None and (t.shape != (N, G) or not t.is_contiguous()):
        raise TypeError(f"{name} must be dense [{N}, {G}]")
    return _address(t, torch.float32, name)


def dvdq_group_norm(X: torch.Tensor, G: int, gamma: Optional[torch.Tensor], beta: Optional[torch.Tensor], eps: float, act: int,
                    Y: torch.Tensor, mean: Optional[torch.Tensor], rstd: Optional[torch.Tensor], workspace: torch.Tensor,
                    stream=None) -> None:
    """Y = act(group norm of X [N, S, C]) over G groups of neighbouring channels, channels last (places of a feature map
    flattened to S); mean and rstd, if given, receive fp32 [N, G] for dvdq_group_norm_backward."""
    dt = X.dtype
    code = _element_type(X, "X", _ANY_FLOAT)
    if X.dim() != 3:
        raise TypeError("X must be [N, S, C]")
    N, S, channels = X.shape
    x, xn, xs = _places(X, dt, X.shape, "X")
    y, yn, ys = _places(Y, dt, X.shape, "Y")
    ga, be, param_code = _norm_params(gamma, beta, dt, code, channels)
    ws, room = _room(workspace)
    _check(load().dvdq_group_norm(x, xn, xs, N, S, channels, G, ga, be, param_code, eps, act, y, yn, ys, _group_stats(mean, N, G, "mean"),
                                  _group_stats(rstd, N, G, "rstd"), code, ws, room, _raw_stream(stream, X)), "dvdq_group_norm")


def dvdq_group_norm_backward(dY: torch.Tensor, X: torch.Tensor, mean: torch.Tensor, rstd: torch.Tensor, G: int,
                             gamma: Optional[torch.Tensor], beta: Optional[torch.Tensor], act: int, dX: Optional[torch.Tensor],
                             dgamma: Optional[torch.Tensor], dbeta: Optional[torch.Tensor], workspace: torch.Tensor,
                             stream=None) -> None:
    """Gradients of dvdq_group_norm: dX (X's type), dgamma and dbeta (fp32 [C]), each written if given."""
    dt = X.dtype
    code = _element_type(X, "X", _ANY_FLOAT)
    if X.dim() != 3:
        raise TypeError("X must be [N, S, C]")
    N, S, channels = X.shape
    x, xn, xs = _places(X, dt, X.shape, "X")
    d, dn, ds = _places(dY, dt, X.shape, "dY")
    y, yn, ys = _places(dX, dt, X.shape, "dX")
    ga, be, param_code = _norm_params(gamma, beta, dt, code, channels)
    ws, room = _room(workspace)
    _check(load().dvdq_group_norm_backward(d, dn, ds, x, xn, xs, _group_stats(mean, N, G, "mean"), _group_stats(rstd, N, G, "rstd"), N, S,
                                           channels, G, ga, be, param_code, act, y, yn, ys, _vector(dgamma, torch.float32, channels, "dgamma"),
                                           _vector(dbeta, torch.float32, channels, "dbeta"), code, ws, room, _raw_stream(stream, X)),
           "dvdq_group_norm_backward")


# Argument structs of include/dvdq.h, packed in one go: ctypes converts arguments one by one, a tenth of a microsecond each.
RMS_NORM_ARGS = struct.Struct("21qiif4x")
RMS_NORM_BACKWARD_ARGS = struct.Struct("20qii")
LINEAR_INT8_ARGS = struct.Struct("16qii")


def _current(t: torch.Tensor, name: str) -> int:
    """The current device, which the calls run on; a tensor that is elsewhere is refused."""
    dev = t.get_device()
    if dev < 0:
        raise TypeError(f"{name} must be a CUDA tensor")
    if dev != torch._C._cuda_getDevice():
        raise ValueError(f"{name} is on {t.device}, the current device is cuda:{torch.cuda.current_device()}")
    return dev


def _refuse(t: torch.Tensor, dtype, shape, dev: int, name: str, inner: str):
    if t.get_device() != dev:
        raise ValueError(f"{name} must be on cuda:{dev} as the others are, got {t.device}")
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.shape != shape:
        raise TypeError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    raise TypeError(f"{name} must {inner}")


# The checks below look at a tensor once, in the order of what is cheap, and say what is wrong afterwards: a call of the smallest
# rows takes longer here than on the GPU.
def _rows3(t: torch.Tensor, dtype, shape, dev: int, name: str):
    """(address, outer pitch, row pitch) of rows in an [N, S, C] tensor, or (N = 1) in an [S, C] one."""
    if t.get_device() == dev and t.dtype is dtype and t.shape == shape:
        st = t.stride()
        if st[-1] == 1 or shape[-1] == 1:
            return (t.data_ptr(), st[0], st[1]) if len(st) == 3 else (t.data_ptr(), 0, st[0])
    _refuse(t, dtype, shape, dev, name, "have unit stride inside a row")


def _dense(t: torch.Tensor, dtype, shape, dev: int, name: str) -> int:
    if t.get_device() == dev and t.dtype is dtype and t.shape == shape and t.is_contiguous():
        return t.data_ptr()
    _refuse(t, dtype, shape, dev, name, "be dense")


def _pitched(t: torch.Tensor, dtype, shape, dev: int, name: str):
    """(address, row pitch) of a matrix with unit inner stride."""
    if t.get_device() == dev and t.dtype is dtype and t.shape == shape:
        pitch, inner = t.stride()
        if inner == 1 or shape[1] == 1:
            return t.data_ptr(), pitch
    _refuse(t, dtype, shape, dev, name, "have unit inner stride")


def _scratch(t: Optional[torch.Tensor], dev: int):
    if t is None:
        return 0, 0
    if t.get_device() != dev or t.dtype is not torch.uint8:
        _refuse(t, torch.uint8, t.shape, dev, "workspace", "be bytes")
    return t.data_ptr(), t.numel()


_NO_ROWS = (0, 0, 0)


def _stream_of(stream, dev: int) -> int:
    return torch._C._cuda_getCurrentRawStream(dev) if stream is None else stream.cuda_stream


def _rows_shape(t: torch.Tensor, name: str):
    shape = t.shape
    if len(shape) == 3:
        return shape, *shape
    if len(shape) == 2:
        return shape, 1, *shape
    raise TypeError(f"{name} must be [S, C] or [N, S, C]")


def _gamma(t: Optional[torch.Tensor], dt, code: int, channels: int, dev: int):
    if t is None:
        return 0, code
    pt = t.dtype
    if pt is not dt and pt is not torch.float32:
        raise TypeError(f"gamma must be {dt} or torch.float32, got {pt}")
    return _dense(t, pt, (channels,), dev, "gamma"), code if pt is dt else F32


def dvdq_rms_norm(X: torch.Tensor, residual: Optional[torch.Tensor], gamma: Optional[torch.Tensor], eps: float,
                  H: Optional[torch.Tensor] = None, Y: Optional[torch.Tensor] = None, codes: Optional[torch.Tensor] = None,
                  scales: Optional[torch.Tensor] = None, rstd: Optional[torch.Tensor] = None, stream=None) -> None:
    """h = X + residual and y = h / sqrt(mean h^2 + eps) * gamma, row by row, for X [S, C] or [N, S, C] (any strides of rows: heads inside a
    fused projection's output).  Written where given: H (h), Y (y), codes int8 with scales fp32 (y in 8 bits, a scale for each row), rstd
    fp32 for dvdq_rms_norm_backward.  H and Y may each be X or residual itself."""
    dt = X.dtype
    code = _element_type(X, "X", _ANY_FLOAT)
    shape, N, S, channels = _rows_shape(X, "X")
    dev = _current(X, "X")
    x = _rows3(X, dt, shape, dev, "X")
    r = _rows3(residual, dt, shape, dev, "residual") if residual is not None else _NO_ROWS
    h = _rows3(H, dt, shape, dev, "H") if H is not None else _NO_ROWS
    y = _rows3(Y, dt, shape, dev, "Y") if Y is not None else _NO_ROWS
    c = _rows3(codes, torch.int8, shape, dev, "codes") if codes is not None else _NO_ROWS
    s = _dense(scales, torch.float32, shape[:-1], dev, "scales") if scales is not None else 0
    q = _dense(rstd, torch.float32, shape[:-1], dev, "rstd") if rstd is not None else 0
    ga, param_code = _gamma(gamma, dt, code, channels, dev)
    args = RMS_NORM_ARGS.pack(*x, *r, *h, *y, *c, N, S, channels, ga, s, q, param_code, code, eps)
    status = load().dvdq_rms_norm(args, _stream_of(stream, dev))
    if status:
        raise DvdqError(status, "dvdq_rms_norm")


def dvdq_rms_norm_backward_workspace_bytes(N: int, S: int, C_: int) -> int:
    return int(load().dvdq_rms_norm_backward_workspace_bytes(N, S, C_))


def dvdq_rms_norm_backward(dY: torch.Tensor, H: torch.Tensor, rstd: torch.Tensor, gamma: Optional[torch.Tensor], dH: Optional[torch.Tensor],
                           dX: Optional[torch.Tensor], dgamma: Optional[torch.Tensor], workspace: Optional[torch.Tensor] = None,
                           stream=None) -> None:
    """Gradients of dvdq_rms_norm: dX (of X and of the residual alike; dH, if given, is added: the gradient that reaches h along the residual stream)
    and dgamma (fp32 [C]), each written if given.  H: the h of the forward call.  dX may be dY, H or dH itself.  The workspace is needed for dgamma."""
    dt = H.dtype
    code = _element_type(H, "H", _ANY_FLOAT)
    shape, N, S, channels = _rows_shape(H, "H")
    dev = _current(H, "H")
    h = _rows3(H, dt, shape, dev, "H")
    d = _rows3(dY, dt, shape, dev, "dY")
    e = _rows3(dH, dt, shape, dev, "dH") if dH is not None else _NO_ROWS
    x = _rows3(dX, dt, shape, dev, "dX") if dX is not None else _NO_ROWS
    q = _dense(rstd, torch.float32, shape[:-1], dev, "rstd")
    ga, param_code = _gamma(gamma, dt, code, channels, dev)
    dg = _dense(dgamma, torch.float32, (channels,), dev, "dgamma") if dgamma is not None else 0
    args = RMS_NORM_BACKWARD_ARGS.pack(*d, *h, *e, *x, N, S, channels, ga, q, dg, *_scratch(workspace, dev), param_code, code)
    status = load().dvdq_rms_norm_backward(args, _stream_of(stream, dev))
    if status:
        raise DvdqError(status, "dvdq_rms_norm_backward")


def dvdq_quantize_rows(X: torch.Tensor, codes: torch.Tensor, scales: torch.Tensor, stream=None) -> None:
    """codes int8 [M, K] = round(X / scale) with scale = max |row| / 127 (scales fp32 [M]): operands of dvdq_linear_int8."""
    code = _element_type(X, "X", _ANY_FLOAT)
    shape = X.shape
    if len(shape) != 2:
        raise TypeError("X must be 2-D")
    dev = _current(X, "X")
    x, ldx = _pitched(X, X.dtype, shape, dev, "X")
    c, ldc = _pitched(codes, torch.int8, shape, dev, "codes")
    M, K = shape
    _check(load().dvdq_quantize_rows(x, M, K, ldx, c, ldc, _dense(scales, torch.float32, (M,), dev, "scales"), code, _stream_of(stream, dev)),
           "dvdq_quantize_rows")


def dvdq_linear_int8_workspace_bytes(M: int, N: int, K: int) -> int:
    return int(load().dvdq_linear_int8_workspace_bytes(M, N, K))


def dvdq_linear_int8(A: torch.Tensor, a_scales: torch.Tensor, W: torch.Tensor, w_scales: torch.Tensor, bias: Optional[torch.Tensor],
                     residual: Optional[torch.Tensor], act: int, Y: torch.Tensor, workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """Y = act(a_scales w_scales^T * (A W^T) + bias) + residual for int8 codes A [M, K] and W [N, K] with a scale for each row; Y, bias and residual
    in bf16 or fp16.  residual may be Y itself.  Rows start on 16 bytes; workspace: dvdq_linear_int8_workspace_bytes(M, N, K) bytes, None
    where that is 0."""
    dt = Y.dtype
    code = _element_type(Y, "Y", _HALF_FLOAT)
    a_shape, w_shape = A.shape, W.shape
    if len(a_shape) != 2 or len(w_shape) != 2 or a_shape[1] != w_shape[1]:
        raise TypeError(f"A and W must be [M, K] and [N, K], got {tuple(a_shape)} and {tuple(w_shape)}")
    (M, K), N = a_shape, w_shape[0]
    dev = _current(A, "A")
    y_shape = (M, N)
    args = LINEAR_INT8_ARGS.pack(
        *_pitched(A, torch.int8, a_shape, dev, "A"), *_pitched(W, torch.int8, w_shape, dev, "W"),
        _dense(a_scales, torch.float32, (M,), dev, "a_scales"), _dense(w_scales, torch.float32, (N,), dev, "w_scales"),
        _dense(bias, dt, (N,), dev, "bias") if bias is not None else 0,
        *(_pitched(residual, dt, y_shape, dev, "residual") if residual is not None else (0, 0)), *_pitched(Y, dt, y_shape, dev, "Y"),
        M, N, K, *_scratch(workspace, dev), act, code)
    status = load().dvdq_linear_int8(args, _stream_of(stream, dev))
    if status:
        raise DvdqError(status, "dvdq_linear_int8")


# ------------------------------------------------------------------ test / debug entry points

def dvdq_qgemm_int32(codes: torch.Tensor, code_sums: torch.Tensor, M: int, q: ActQuant, w: Weights,
                     acc: torch.Tensor, stream=None) -> None:
    ld = _row_major(acc, "acc")
    _check(load().dvdq_qgemm_int32(_ptr(codes, torch.uint8, "codes"), _ptr(code_sums, torch.int32, "code_sums"),
                                   M, C.byref(q), C.byref(w), _ptr(acc, torch.int32, "acc"), ld, _stream(stream)),
           "dvdq_qgemm_int32")


def dvdq_pack_act_codes(codes_nat: torch.Tensor, q: ActQuant, codes: torch.Tensor, code_sums: torch.Tensor,
                        stream=None) -> None:
    M, K = codes_nat.shape
    if not codes_nat.is_contiguous():
        raise TypeError("codes_nat must be contiguous")
    _check(load().dvdq_pack_act_codes(_ptr(codes_nat, torch.int8, "codes_nat"), M, K, C.byref(q),
                                      _ptr(codes, torch.uint8, "codes"), _ptr(code_sums, torch.int32, "code_sums"),
                                      _stream(stream)), "dvdq_pack_act_codes")


def dvdq_unpack_act_codes(codes: torch.Tensor, M: int, K: int, q: ActQuant, codes_nat: torch.Tensor,
                          stream=None) -> None:
    if not codes_nat.is_contiguous() or tuple(codes_nat.shape) != (M, K):
        raise TypeError("codes_nat must be contiguous [M, K]")
    _check(load().dvdq_unpack_act_codes(_ptr(codes, torch.uint8, "codes"), M, K, C.byref(q),
                                        _ptr(codes_nat, torch.int8, "codes_nat"), _stream(stream)),
           "dvdq_unpack_act_codes")


def dvdq_unpack_weights(w: Weights, Wq: torch.Tensor, delta: torch.Tensor, zero: torch.Tensor, stream=None) -> None:
    if not Wq.is_contiguous():
        raise TypeError("Wq must be contiguous")
    _check(load().dvdq_unpack_weights(C.byref(w), _ptr(Wq, torch.uint8, "Wq"), _ptr(delta, torch.float32, "delta"),
                                      _ptr(zero, torch.int32, "zero"), _stream(stream)), "dvdq_unpack_weights")


def dvdq_rotate_weights(W: torch.Tensor, rot_block: int, W_rot: torch.Tensor, stream=None) -> None:
    """W~ = W R along K: bf16 [N, K] -> dense fp32 [N, K]."""
    ldw = _row_major(W, "W")
    N, K = W.shape
    if not W_rot.is_contiguous() or tuple(W_rot.shape) != (N, K):
        raise TypeError("W_rot must be dense [N, K]")
    _check(load().dvdq_rotate_weights(_ptr(W, torch.bfloat16, "W"), N, K, ldw, rot_block,
                                      _ptr(W_rot, torch.float32, "W_rot"), _stream(stream)), "dvdq_rotate_weights")


def dvdq_quantize_weights_symmetric(W: torch.Tensor, rot_block: int, blob: torch.Tensor, stream=None) -> Weights:
    """bf16 [N, K] weights -> rotated, symmetric 4-bit codes (z = 8, Delta = absmax / 7) in a blob."""
    ldw = _row_major(W, "W")
    N, K = W.shape
    w = Weights()
    _check(load().dvdq_quantize_weights_symmetric(_ptr(W, torch.bfloat16, "W"), N, K, ldw, rot_block,
                                                  _ptr(blob, torch.uint8, "blob"), C.byref(w), _stream(stream)),
           "dvdq_quantize_weights_symmetric")
    return w


def dvdq_weight_operand_bytes(N: int, K: int) -> int:
    return int(load().dvdq_weight_operand_bytes(N, K))


def dvdq_widen_weights(w: Weights, operand: torch.Tensor, stream=None) -> Weights:
    """Writes the 4-bit codes of `w` one int8 each into `operand` (uint8, >= N * K bytes) and returns
    a handle that refers to both; GEMMs given it read the weight operand with TMA."""
    out = Weights()
    _check(load().dvdq_widen_weights(C.byref(w), _ptr(operand, torch.uint8, "operand"), operand.numel(), C.byref(out),
                                     _stream(stream)), "dvdq_widen_weights")
    return out


def dvdq_int8_mma_ceiling(iters: int, stream=None) -> int:
    """Launches the int8 tensor-pipe issue loop; returns the integer operations of the launch."""
    ops = C.c_int64(0)
    _check(load().dvdq_int8_mma_ceiling(iters, C.byref(ops), _stream(stream)), "dvdq_int8_mma_ceiling")
    return int(ops.value)


def dvdq_debug_wait_timeout(limit_ns: int, stream=None) -> None:
    _check(load().dvdq_debug_wait_timeout(int(limit_ns), _stream(stream)), "dvdq_debug_wait_timeout")


def dvdq_bgr_quantize(W_rot: torch.Tensor, n_steps: int, eps: float, max_iter: int, Wq: torch.Tensor,
                      delta: torch.Tensor, zero: torch.Tensor, stream=None) -> None:
    """Bounded-init Grid Refinement of rotated fp32 weights [N, K] -> (Wq uint8, delta fp32, zero int32)."""
    if W_rot.dim() != 2 or not W_rot.is_contiguous() or not Wq.is_contiguous():
        raise TypeError("W_rot and Wq must be dense [N, K]")
    N, K = W_rot.shape
    _check(load().dvdq_bgr_quantize(_ptr(W_rot, torch.float32, "W_rot"), N, K, n_steps, float(eps), max_iter,
                                    _ptr(Wq, torch.uint8, "Wq"), _ptr(delta, torch.float32, "delta"),
                                    _ptr(zero, torch.int32, "zero"), _stream(stream)), "dvdq_bgr_quantize")


def dvdq_gbs_l1_terms(F_t: torch.Tensor, F_prev: torch.Tensor, terms: torch.Tensor, stream=None) -> None:
    """terms (float64[2], device) <- (||F_t - F_prev||_1, ||F_prev||_1) of two bf16 tensors of equal size."""
    if F_t.numel() != F_prev.numel() or not F_t.is_contiguous() or not F_prev.is_contiguous():
        raise TypeError("F_t and F_prev must be contiguous and of equal size")
    if terms.dtype != torch.float64 or terms.numel() < 2:
        raise TypeError("terms must hold two float64 values")
    _check(load().dvdq_gbs_l1_terms(_ptr(F_t, torch.bfloat16, "F_t"), _ptr(F_prev, torch.bfloat16, "F_prev"), F_t.numel(),
                                    _ptr(terms, torch.float64, "terms"), _stream(stream)), "dvdq_gbs_l1_terms")


def dvdq_gbs_init(delta: float, b_low: int, b_high: int) -> GbsState:
    g = GbsState()
    _check(load().dvdq_gbs_init(C.byref(g), float(delta), b_low, b_high), "dvdq_gbs_init")
    return g


def dvdq_gbs_next_bits(g: GbsState) -> int:
    return int(load().dvdq_gbs_next_bits(C.byref(g)))


def dvdq_gbs_observe(g: GbsState, l1_change: float, l1_prev: float) -> None:
    _check(load().dvdq_gbs_observe(C.byref(g), float(l1_change), float(l1_prev)), "dvdq_gbs_observe")


def dvdq_last_device_status():
    """(status, detail) of a device-side failure, (OK, 0) where there is none; synchronizes the device and clears what it
    reports.  One failure a call: the quantized layers' and that of the operators around them are kept apart."""
    d = C.c_uint32(0)
    s = load().dvdq_last_device_status(C.byref(d))
    return int(s), int(d.value)
