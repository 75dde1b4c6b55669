"""Python binding of libtardis (the C ABI in include/tardis.h): argument marshalling only.

Every step of the partially linear FFN forward (TARDIS, arXiv 2501.10054: constant folding,
predictor, speculative folded product, result fixing) runs inside the CUDA library; this
module turns torch tensors into device pointers and status codes into exceptions.  There is
no CPU fallback: importing works anywhere, but any call needs libtardis.so and a CUDA device.
"""
from __future__ import annotations

import ctypes
import operator
import os
import struct
from typing import Optional

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libtardis.so")

TARDIS_OK = 0
TARDIS_F32, TARDIS_BF16 = 0, 1
TARDIS_ACT_GELU_TANH, TARDIS_ACT_GELU_ERF, TARDIS_ACT_RELU = 0, 1, 2
TARDIS_ACT_NONE = -1

EXPORTS = ["tardis_fold", "tardis_ffn_forward", "tardis_ffn_forward_static", "tardis_gemm_bf16", "tardis_linear", "tardis_grouped_linear", "tardis_route", "tardis_stats",
           "tardis_set_debug_capture", "tardis_export_folded", "tardis_set_path", "tardis_set_deterministic", "tardis_stack_forward", "tardis_build_predictor", "tardis_destroy", "tardis_calibrate",
           "tardis_debug_phase_stamps", "tardis_range_search", "tardis_neuron_thresholds", "tardis_debug_wait_timeout", "tardis_clear_error", "tardis_debug_fail_alloc", "tardis_debug_live_allocations", "tardis_debug_damage_guard",
           "tardis_save", "tardis_load", "tardis_status_string", "tardis_last_error"]


class TardisError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(what)


class FoldDesc(ctypes.Structure):
    _fields_ = [("d_model", ctypes.c_int32), ("d_ff", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("act", ctypes.c_int32), ("W1", ctypes.c_void_p), ("W2", ctypes.c_void_p),
                ("b1", ctypes.c_void_p), ("b2", ctypes.c_void_p), ("lo", ctypes.c_void_p),
                ("hi", ctypes.c_void_p), ("a", ctypes.c_void_p), ("c", ctypes.c_void_p),
                ("pred_bits", ctypes.c_int32), ("pred_group", ctypes.c_int32),
                ("pred_codes", ctypes.c_void_p), ("pred_scale", ctypes.c_void_p),
                ("pred_zero", ctypes.c_void_p), ("flags", ctypes.c_uint32)]


class LinearDesc(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int64), ("k", ctypes.c_int32), ("o", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("out_dtype", ctypes.c_int32), ("act", ctypes.c_int32), ("x", ctypes.c_void_p), ("ldx", ctypes.c_int64),
                ("W", ctypes.c_void_p), ("ldw", ctypes.c_int64), ("bias", ctypes.c_void_p), ("residual", ctypes.c_void_p),
                ("ldr", ctypes.c_int64), ("y", ctypes.c_void_p), ("ldy", ctypes.c_int64)]


class GroupedDesc(ctypes.Structure):
    _fields_ = [("n_rows", ctypes.c_int64), ("n_experts", ctypes.c_int32), ("k", ctypes.c_int32), ("o", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("out_dtype", ctypes.c_int32), ("act", ctypes.c_int32), ("x", ctypes.c_void_p),
                ("ldx", ctypes.c_int64), ("n_x", ctypes.c_int64), ("W", ctypes.c_void_p), ("ldw", ctypes.c_int64),
                ("stride_w", ctypes.c_int64), ("bias", ctypes.c_void_p), ("offsets", ctypes.c_void_p), ("rows", ctypes.c_void_p),
                ("residual", ctypes.c_void_p), ("ldr", ctypes.c_int64), ("y", ctypes.c_void_p), ("ldy", ctypes.c_int64),
                ("n_tokens", ctypes.c_int64), ("top_k", ctypes.c_int32), ("slots", ctypes.c_void_p), ("weights", ctypes.c_void_p),
                ("work", ctypes.c_void_p), ("work_bytes", ctypes.c_size_t)]


class Stats(ctypes.Structure):
    _fields_ = [(n, ctypes.c_uint64) for n in
                ("calls", "tokens", "flagged_total", "flagged_max", "last_path", "bytes_folded",
                 "bytes_predictor", "bytes_tables", "bytes_w1", "bytes_w2t", "bytes_scratch",
                 "device_error", "exact_rechecks", "launches", "last_union")]

    def as_dict(self):
        return {n: int(getattr(self, n)) for n, _ in self._fields_}


_lib = None


def load_library(path: Optional[str] = None) -> ctypes.CDLL:
    """Loads libtardis.so (built in-tree by paper_2501_10054_b200.build).  Fails loudly if absent."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    p = path or LIB_PATH
    if not os.path.exists(p):
        raise TardisError(-1, "libtardis.so not found at %s: run `python -m paper_2501_10054_b200.build` "
                              "(there is no CPU fallback)" % p)
    lib = ctypes.CDLL(p)
    vp, i64, i32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32
    lib.tardis_fold.argtypes = [ctypes.POINTER(FoldDesc), vp, ctypes.POINTER(vp)]
    lib.tardis_ffn_forward.argtypes = [vp, vp, vp, i64, vp]
    lib.tardis_ffn_forward_static.argtypes = [vp, vp, vp, i64, vp]
    lib.tardis_stats.argtypes = [vp, ctypes.POINTER(Stats)]
    lib.tardis_set_debug_capture.argtypes = [vp, vp, vp]
    lib.tardis_export_folded.argtypes = [vp, vp, vp, vp]
    lib.tardis_set_path.argtypes = [vp, i32]
    lib.tardis_set_deterministic.argtypes = [vp, i32]
    lib.tardis_build_predictor.argtypes = [i32, i32, i32, vp, vp, i32, i32, vp, vp, vp, vp]
    lib.tardis_stack_forward.argtypes = [vp, vp, vp, vp, ctypes.c_size_t, vp, ctypes.c_size_t, ctypes.c_int64, vp]
    lib.tardis_destroy.argtypes = [vp]
    lib.tardis_gemm_bf16.argtypes = [i32, i32, i32, vp, i32, vp, i32, vp, i32, vp]
    lib.tardis_linear.argtypes = [vp, vp]
    lib.tardis_grouped_linear.argtypes = [vp, vp]
    lib.tardis_route.argtypes = [i64, i32, i32, i32, vp, i64, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
    lib.tardis_calibrate.argtypes = [i32, i32, vp, i64, vp, ctypes.c_double, ctypes.c_double, i32, vp, vp, vp, vp, vp]
    lib.tardis_debug_phase_stamps.argtypes = [vp, i32]
    lib.tardis_range_search.argtypes = [i32, i32, vp, i64, vp, vp, ctypes.c_double, ctypes.c_double, i32, vp, vp, vp, vp, vp, vp]
    lib.tardis_debug_wait_timeout.argtypes = [vp, i64, vp]
    lib.tardis_neuron_thresholds.argtypes = [i32, i32, vp, i64, vp, vp, vp, i32, ctypes.c_double, ctypes.c_double, ctypes.c_double, vp, vp, vp]
    lib.tardis_clear_error.argtypes = [vp]
    lib.tardis_debug_fail_alloc.argtypes = [i32]
    lib.tardis_debug_live_allocations.argtypes = [ctypes.POINTER(i64), ctypes.POINTER(i64)]
    lib.tardis_debug_damage_guard.argtypes = [vp, i32, i32]
    lib.tardis_save.argtypes = [vp, ctypes.c_char_p]
    lib.tardis_load.argtypes = [ctypes.c_char_p, vp, ctypes.POINTER(vp)]
    for name in EXPORTS[:-2]:
        getattr(lib, name).restype = ctypes.c_int
    lib.tardis_status_string.argtypes = [ctypes.c_int]
    lib.tardis_status_string.restype = ctypes.c_char_p
    lib.tardis_last_error.argtypes = []
    lib.tardis_last_error.restype = ctypes.c_char_p
    if path is None:
        _lib = lib
    return lib


def _check(status: int, what: str):
    if status != TARDIS_OK:
        lib = load_library()
        msg = lib.tardis_status_string(status).decode()
        detail = lib.tardis_last_error().decode()
        raise TardisError(status, "%s: %s%s" % (what, msg, (" [" + detail + "]") if detail and status == 4 else ""))


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous():
        raise TardisError(1, "tensors must be contiguous CUDA tensors")
    return t.data_ptr()


def _stream(stream) -> Optional[int]:
    if stream is None:
        stream = torch.cuda.current_stream()
    return stream.cuda_stream or None


def _dtype_code(dt: torch.dtype) -> int:
    if dt == torch.float32:
        return TARDIS_F32
    if dt == torch.bfloat16:
        return TARDIS_BF16
    raise TardisError(1, "dtype must be float32 or bfloat16")


def tardis_fold(W1, W2, lo, hi, a, c, pred_codes, pred_scale, pred_zero, pred_group, b1=None, b2=None,
                act=TARDIS_ACT_GELU_TANH, pred_bits=2, stream=None, flags=0) -> int:
    """tardis_fold of the C ABI.  Returns the opaque handle (an integer)."""
    lib = load_library()
    h, d = W1.shape
    desc = FoldDesc(d, h, _dtype_code(W1.dtype), act, _ptr(W1), _ptr(W2), _ptr(b1), _ptr(b2), _ptr(lo), _ptr(hi),
                    _ptr(a), _ptr(c), pred_bits, pred_group, _ptr(pred_codes), _ptr(pred_scale), _ptr(pred_zero), flags)
    out = ctypes.c_void_p()
    _check(lib.tardis_fold(ctypes.byref(desc), _stream(stream), ctypes.byref(out)), "tardis_fold")
    return out.value


def tardis_ffn_forward(handle: int, x: torch.Tensor, y: torch.Tensor, n_tokens: Optional[int] = None, stream=None):
    lib = load_library()
    n = x.shape[0] if n_tokens is None else n_tokens
    _check(lib.tardis_ffn_forward(handle, _ptr(x), _ptr(y), n, _stream(stream)), "tardis_ffn_forward")
    return y


def tardis_ffn_forward_static(handle: int, x: torch.Tensor, y: torch.Tensor, n_tokens: Optional[int] = None, stream=None):
    """tardis_ffn_forward_static of the C ABI: the same forward for callers that may not allocate device
    memory; its scratch is a fixed array inside the library (at most 64 tokens, 4 MiB of scratch)."""
    lib = load_library()
    n = x.shape[0] if n_tokens is None else n_tokens
    st = lib.tardis_ffn_forward_static(handle, _ptr(x), _ptr(y), n, _stream(stream))
    if st == 2:
        raise TardisError(st, "tardis_ffn_forward_static: %s" % lib.tardis_last_error().decode())
    _check(st, "tardis_ffn_forward_static")
    return y


def tardis_gemm_bf16(A: torch.Tensor, B: torch.Tensor, C: torch.Tensor, stream=None):
    """C[M, N] (float32) = A[M, K] B[N, K]^T for bfloat16 row-major A, B (last stride 1)."""
    lib = load_library()
    M, K = A.shape
    N = B.shape[0]
    if A.stride(1) != 1 or B.stride(1) != 1 or C.stride(1) != 1 or not (A.is_cuda and B.is_cuda and C.is_cuda):
        raise TardisError(1, "tensors must be CUDA tensors with unit inner stride")
    _check(lib.tardis_gemm_bf16(M, N, K, A.data_ptr(), A.stride(0), B.data_ptr(), B.stride(0), C.data_ptr(), C.stride(0),
                                _stream(stream)), "tardis_gemm_bf16")
    return C


# The descriptors of tardis_linear and tardis_grouped_linear as packed bytes (native alignment, as LinearDesc and GroupedDesc): a call that is over in
# a few microseconds on the device should not take longer to describe.
_PACK_LINEAR = struct.Struct("@qiiiiiPqPqPPqPq").pack
_PACK_GROUPED = struct.Struct("@qiiiiiiPqqPqqPPPPqPqqiPPPN").pack
_ACTS = (TARDIS_ACT_NONE, TARDIS_ACT_GELU_TANH, TARDIS_ACT_GELU_ERF, TARDIS_ACT_RELU)


def _whole(v, name: str) -> int:
    try:
        return operator.index(v)
    except TypeError:
        raise TardisError(1, "%s must be a whole number" % name) from None


def _check_act(act) -> None:
    if _whole(act, "act") not in _ACTS:
        raise TardisError(1, "act must be TARDIS_ACT_NONE, TARDIS_ACT_GELU_TANH, TARDIS_ACT_GELU_ERF or TARDIS_ACT_RELU")


def _current(x: torch.Tensor) -> int:
    """The index of x's device, which has to be the current one: that is where the launch goes."""
    index = x.get_device()
    if index < 0 or index != torch.cuda.current_device():
        raise TardisError(1, "tensors must lie on the current CUDA device")
    return index


def _matrix(t: torch.Tensor, name: str, dtype, rows: int, cols: int, index: int):
    """(data pointer, leading dimension) of a matrix with unit inner stride."""
    shape, strides = t.shape, t.stride()
    if len(shape) != 2:
        raise TardisError(1, "%s must be a matrix" % name)
    ld, unit = strides
    if t.dtype is not dtype or shape[0] != rows or shape[1] != cols or t.get_device() != index or (unit != 1 and cols > 1):
        raise TardisError(1, "%s must be a %s matrix of %d x %d on the same device with unit inner stride" % (name, dtype, rows, cols))
    return t.data_ptr(), ld if rows > 1 else cols


def _vector(t: Optional[torch.Tensor], name: str, dtype, shape, index: int) -> int:
    if t is None:
        return 0
    if t.dtype is not dtype or t.shape != shape or t.get_device() != index or not t.is_contiguous():
        raise TardisError(1, "%s must be a contiguous %s tensor of shape %s on the same device" % (name, dtype, shape))
    return t.data_ptr()


def _raw_stream(stream, index: int) -> int:
    return torch._C._cuda_getCurrentRawStream(index) if stream is None else stream.cuda_stream


def _empty(x: torch.Tensor, shape, dtype, stream, zero: bool = False) -> torch.Tensor:
    """Memory for a call on `stream`: taken from that stream's own, which nothing that is still under way on the current one uses."""
    make = x.new_zeros if zero else x.new_empty
    if stream is None:
        return make(shape, dtype=dtype)
    with torch.cuda.stream(stream):
        return make(shape, dtype=dtype)


def tardis_linear(x: torch.Tensor, W: torch.Tensor, bias: Optional[torch.Tensor] = None, act: int = TARDIS_ACT_NONE,
                  residual: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None, out_dtype=None, stream=None):
    """y = act(x W^T + bias) + residual in one launch (see tardis_linear in tardis.h): x [n, k], W [o, k] float32 or bfloat16
    with unit inner stride, bias [o] float32, residual and y [n, o] in out_dtype (x's dtype, or float32).  Returns y (`out`
    when given; it may be the residual).  No gradient is recorded, here and in the calls below."""
    if x.dim() != 2 or W.dim() != 2 or W.shape[1] != x.shape[1]:
        raise TardisError(1, "x must be [n, k] and W [o, k]")
    _check_act(act)
    index, dtype = _current(x), x.dtype
    (n, k), o = x.shape, W.shape[0]
    if out_dtype is None:
        out_dtype = dtype if out is None else out.dtype
    code, out_code = _dtype_code(dtype), _dtype_code(out_dtype)
    if out is None:
        out = _empty(x, (n, o), out_dtype, stream)
    px, ldx = _matrix(x, "x", dtype, n, k, index)
    pw, ldw = _matrix(W, "W", dtype, o, k, index)
    py, ldy = _matrix(out, "out", out_dtype, n, o, index)
    pr, ldr = _matrix(residual, "residual", out_dtype, n, o, index) if residual is not None else (0, 0)
    desc = _PACK_LINEAR(n, k, o, code, out_code, act, px, ldx, pw, ldw, _vector(bias, "bias", torch.float32, (o,), index), pr, ldr, py, ldy)
    status = load_library().tardis_linear(desc, _raw_stream(stream, index))
    if status != TARDIS_OK:
        _check(status, "tardis_linear")
    return out


def _grouped(x, W, offsets, bias, act, rows, residual, out, out_dtype, back, work, stream, what):
    if x.dim() != 2 or W.dim() != 3 or W.shape[2] != x.shape[1]:
        raise TardisError(1, "x must be [n, k] and W [experts, o, k]")
    _check_act(act)
    index, dtype, i32 = _current(x), x.dtype, torch.int32
    (nx, k), (experts, o, _) = x.shape, W.shape
    n = nx if rows is None else rows.numel()
    if out_dtype is None:
        out_dtype = dtype if out is None else out.dtype
    code, out_code = _dtype_code(dtype), _dtype_code(out_dtype)
    tokens = top_k = room = ps = pc = pwork = 0
    n_out = n
    if back is not None:
        slots, weights = back
        if slots.dim() != 2:
            raise TardisError(1, "slots must be [tokens, top_k]")
        tokens, top_k = slots.shape
        ps, pc = _vector(slots, "slots", i32, (tokens, top_k), index), _vector(weights, "weights", torch.float32, (tokens, top_k), index)
        n_out, room = tokens, 4 * n * ((o + 7) // 8 * 8)
        if work is None:
            work = _empty(x, (room // 4,), torch.float32, stream)
        elif work.get_device() != index or not work.is_contiguous() or work.numel() * work.element_size() < room:
            raise TardisError(1, "work must be a contiguous tensor of at least 4 rows o bytes (o rounded up to 8) on x's device")
        pwork = work.data_ptr()
    elif rows is not None and n >= 1024 and o >= 4096 and k <= 1 << 17 and dtype is torch.bfloat16 and out_dtype is torch.bfloat16:      # (where long calls use it)
        work, room = _empty(x, (n, k), dtype, stream), 2 * n * k
        pwork = work.data_ptr()
    if out is None:                                          # (rows in no group are left as they were: zero)
        out = _empty(x, (n_out, o), out_dtype, stream, zero=back is None)
    px, ldx = _matrix(x, "x", dtype, nx, k, index)
    stride_w, ldw, unit = W.stride()
    if W.dtype is not dtype or W.get_device() != index or unit != 1:
        raise TardisError(1, "W must have x's dtype and device and unit inner stride")
    py, ldy = _matrix(out, "out", out_dtype, n_out, o, index)
    pr, ldr = _matrix(residual, "residual", out_dtype, n_out, o, index) if residual is not None else (0, 0)
    desc = _PACK_GROUPED(n, experts, k, o, code, out_code, act, px, ldx, nx, W.data_ptr(), ldw if o > 1 else k, stride_w,
                         _vector(bias, "bias", torch.float32, (experts, o), index), _vector(offsets, "offsets", i32, (experts + 1,), index),
                         _vector(rows, "rows", i32, (n,), index), pr, ldr, py, ldy, tokens, top_k, ps, pc, pwork, room)
    status = load_library().tardis_grouped_linear(desc, _raw_stream(stream, index))
    if status != TARDIS_OK:
        _check(status, what)
    return out


def tardis_grouped_linear(x: torch.Tensor, W: torch.Tensor, offsets: torch.Tensor, bias: Optional[torch.Tensor] = None,
                          act: int = TARDIS_ACT_NONE, rows: Optional[torch.Tensor] = None, residual: Optional[torch.Tensor] = None,
                          out: Optional[torch.Tensor] = None, out_dtype=None, stream=None):
    """The product of tardis_linear with each group's own weights (see tardis_grouped_linear in tardis.h): W [experts, o, k], bias
    [experts, o], offsets int32 [experts + 1] on the device; y[r] = act(W_e x[rows[r]] + bias_e) + residual[r] for
    offsets[e] <= r < offsets[e + 1].  Rows of `out` in no group are left as they were; of a result that is made here they are zero (which
    costs a pass over it: programs that read rows in groups only, as the return to the tokens does, bring `out`)."""
    return _grouped(x, W, offsets, bias, act, rows, residual, out, out_dtype, None, None, stream, "tardis_grouped_linear")


def tardis_grouped_linear_combine(x: torch.Tensor, W: torch.Tensor, offsets: torch.Tensor, slots: torch.Tensor, weights: torch.Tensor,
                                  bias: Optional[torch.Tensor] = None, act: int = TARDIS_ACT_NONE, rows: Optional[torch.Tensor] = None,
                                  residual: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None, out_dtype=None,
                                  work: Optional[torch.Tensor] = None, stream=None):
    """tardis_grouped_linear and the weighted return to the tokens: y[t] = residual[t] + sum_c weights[t, c] f[slots[t, c]], slots int32
    and weights float32 [tokens, top_k].  `work` is scratch of 4 rows o bytes, o rounded up to a multiple of 8 (made here when not given)."""
    return _grouped(x, W, offsets, bias, act, rows, residual, out, out_dtype, (slots, weights), work, stream,
                    "tardis_grouped_linear_combine")


def tardis_route(logits: torch.Tensor, top_k: int, normalise: bool = True, stream=None):
    """The experts of every token (see tardis_route in tardis.h): logits float32 [tokens, experts] with unit inner stride.  Returns
    (experts int32 [tokens, top_k], weights float32 [tokens, top_k], offsets int32 [experts + 1], rows int32 [tokens top_k],
    slots int32 [tokens, top_k]): what tardis_grouped_linear and tardis_grouped_linear_combine take."""
    if logits.dim() != 2:
        raise TardisError(1, "logits must be [tokens, experts]")
    index = _current(logits)
    n, e = logits.shape
    pl, ldl = _matrix(logits, "logits", torch.float32, n, e, index)
    top_k = _whole(top_k, "top_k")
    if not 1 <= top_k <= e:
        raise TardisError(1, "top_k must be between 1 and the number of experts")
    i32 = torch.int32
    experts, slots, rows, weights = _empty(logits, (4, n, top_k), i32, stream).unbind(0)       # (one allocation)
    rows, weights = rows.view(-1), weights.view(torch.float32)
    offsets = _empty(logits, (e + 1,), i32, stream)
    work = _empty(logits, (1024 * e,), i32, stream) if n > 128 else None
    status = load_library().tardis_route(n, e, top_k, 1 if normalise else 0, pl, ldl, experts.data_ptr(), weights.data_ptr(),
                                         offsets.data_ptr(), rows.data_ptr(), slots.data_ptr(), work.data_ptr() if work is not None else 0,
                                         4096 * e if work is not None else 0, _raw_stream(stream, index))
    if status != TARDIS_OK:
        _check(status, "tardis_route")
    return experts, weights, offsets, rows, slots


def tardis_calibrate(z: torch.Tensor, b1: Optional[torch.Tensor], q_lo: float, q_hi: float, act: int, stream=None):
    """Per-neuron ranges and linear fits from calibration pre-activations z[d_ff, n_cal] (float32, CUDA, unit inner
    stride): returns (lo, hi, a, c), float32 tensors of d_ff elements on z's device."""
    if z.dtype != torch.float32 or not z.is_cuda or z.stride(1) != 1:
        raise TardisError(1, "z must be a float32 CUDA tensor with unit inner stride")
    h, n = z.shape
    out = [torch.empty(h, dtype=torch.float32, device=z.device) for _ in range(4)]
    _check(load_library().tardis_calibrate(h, n, z.data_ptr(), z.stride(0), _ptr(b1), float(q_lo), float(q_hi), int(act),
                                           out[0].data_ptr(), out[1].data_ptr(), out[2].data_ptr(), out[3].data_ptr(),
                                           _stream(stream)), "tardis_calibrate")
    return tuple(out)


def tardis_range_search(z: torch.Tensor, b1: Optional[torch.Tensor], threshold, step: float, act: int, stream=None, want_steps=False):
    """Algorithm 1's greedy range search per neuron from calibration pre-activations z[d_ff, n_cal] (float32, CUDA, unit
    inner stride, n_cal <= 2048): returns (lo, hi, a, c) (and the step counts with want_steps).  `threshold` is a float
    (one coverage for all neurons) or a float32 CUDA tensor of d_ff per-neuron thresholds."""
    if z.dtype != torch.float32 or not z.is_cuda or z.stride(1) != 1:
        raise TardisError(1, "z must be a float32 CUDA tensor with unit inner stride")
    h, n = z.shape
    out = [torch.empty(h, dtype=torch.float32, device=z.device) for _ in range(4)]
    steps = torch.zeros(h, dtype=torch.int32, device=z.device) if want_steps else None
    thr_t = threshold if isinstance(threshold, torch.Tensor) else None
    _check(load_library().tardis_range_search(h, n, z.data_ptr(), z.stride(0), _ptr(b1), _ptr(thr_t),
                                              0.0 if thr_t is not None else float(threshold), float(step), int(act),
                                              out[0].data_ptr(), out[1].data_ptr(), out[2].data_ptr(), out[3].data_ptr(),
                                              _ptr(steps), _stream(stream)), "tardis_range_search")
    return tuple(out) + ((steps,) if want_steps else ())


def tardis_neuron_thresholds(z: torch.Tensor, b1: Optional[torch.Tensor], lo: torch.Tensor, hi: torch.Tensor, act: int,
                             t_layer: float, t_min: float, t_max: float, stream=None):
    """Per-neuron coverage thresholds of Section 5.1.1 from the neurons' approximation errors inside [lo, hi): returns
    (err, thresholds), float32 tensors of d_ff elements (see tardis_neuron_thresholds in tardis.h)."""
    if z.dtype != torch.float32 or not z.is_cuda or z.stride(1) != 1:
        raise TardisError(1, "z must be a float32 CUDA tensor with unit inner stride")
    h, n = z.shape
    err = torch.empty(h, dtype=torch.float32, device=z.device)
    thr = torch.empty(h, dtype=torch.float32, device=z.device)
    _check(load_library().tardis_neuron_thresholds(h, n, z.data_ptr(), z.stride(0), _ptr(b1), _ptr(lo), _ptr(hi), int(act),
                                                   float(t_layer), float(t_min), float(t_max), _ptr(err), _ptr(thr),
                                                   _stream(stream)), "tardis_neuron_thresholds")
    return err, thr


def tardis_stats(handle: int) -> dict:
    lib = load_library()
    st = Stats()
    _check(lib.tardis_stats(handle, ctypes.byref(st)), "tardis_stats")
    return st.as_dict()


def tardis_set_debug_capture(handle: int, flag_bitmap: Optional[torch.Tensor], scores: Optional[torch.Tensor]):
    _check(load_library().tardis_set_debug_capture(handle, _ptr(flag_bitmap), _ptr(scores)), "tardis_set_debug_capture")


def tardis_export_folded(handle: int, Wf: Optional[torch.Tensor], bf: Optional[torch.Tensor], stream=None):
    _check(load_library().tardis_export_folded(handle, _ptr(Wf), _ptr(bf), _stream(stream)), "tardis_export_folded")


def tardis_set_path(handle: int, path: int):
    _check(load_library().tardis_set_path(handle, path), "tardis_set_path")


def tardis_set_deterministic(handle: int, on: bool):
    _check(load_library().tardis_set_deterministic(handle, 1 if on else 0), "tardis_set_deterministic")


def tardis_debug_phase_stamps(max_ctas: int = 512):
    """Phase stamps of the most recent fused decode launch as a numpy int64 array [max_ctas, 16] (needs a
    library built with TARDIS_PHASE_STAMPS; the ordinary build raises UNSUPPORTED)."""
    import numpy as np
    buf = np.zeros((max_ctas, 16), dtype=np.int64)
    _check(load_library().tardis_debug_phase_stamps(buf.ctypes.data, max_ctas), "tardis_debug_phase_stamps")
    return buf


def tardis_debug_wait_timeout(handle: int, limit_cycles: int, stream=None):
    """Launches one warp whose bounded wait runs out after limit_cycles SM cycles (testing aid for the time-out report)."""
    _check(load_library().tardis_debug_wait_timeout(handle, int(limit_cycles), _stream(stream)), "tardis_debug_wait_timeout")


def tardis_clear_error(handle: int):
    _check(load_library().tardis_clear_error(handle), "tardis_clear_error")


def tardis_build_predictor(W1: torch.Tensor, U: Optional[torch.Tensor], bits: int, group: int, stream=None):
    """Predictor of a layer by error-compensated quantisation on the GPU (see tardis_build_predictor in tardis.h).
    W1 [h, d] float32 or bfloat16, U [d, d] float64 upper Cholesky factor of the inverse Hessian (None: round to nearest).
    Returns (codes int32 [h, d bits / 32], scale [h, d / group] in W1's dtype, zero uint8 [h, d / group])."""
    h, d = W1.shape
    if not W1.is_contiguous() or (U is not None and (U.dtype != torch.float64 or not U.is_contiguous() or tuple(U.shape) != (d, d))):
        raise TardisError(1, "W1 must be contiguous and U a contiguous float64 [d, d] tensor")
    codes = torch.empty(h, d * bits // 32, dtype=torch.int32, device=W1.device)
    scale = torch.empty(h, d // group, dtype=W1.dtype, device=W1.device)
    zero = torch.empty(h, d // group, dtype=torch.uint8, device=W1.device)
    _check(load_library().tardis_build_predictor(h, d, _dtype_code(W1.dtype), _ptr(W1), _ptr(U), bits, group, _ptr(codes),
                                                 _ptr(scale), _ptr(zero), _stream(stream)), "tardis_build_predictor")
    return codes, scale, zero


class StackDesc(ctypes.Structure):
    _fields_ = [("n_layers", ctypes.c_int32), ("layers", ctypes.POINTER(ctypes.c_void_p)), ("normalise", ctypes.c_int32),
                ("ln_gamma", ctypes.POINTER(ctypes.c_void_p)), ("ln_beta", ctypes.POINTER(ctypes.c_void_p)),
                ("ln_eps", ctypes.c_float), ("residual", ctypes.c_int32)]


def tardis_stack_forward(handles, x: torch.Tensor, y: torch.Tensor, gammas=None, betas=None, eps: float = 1e-5,
                         normalise: bool = True, residual: bool = True, work: Optional[torch.Tensor] = None,
                         keep: Optional[torch.Tensor] = None, stream=None):
    """The layers `handles` chained on one residual stream (see tardis_stack_forward in tardis.h).  `work` is scratch of
    2 n d elements in x's dtype (made here when neither it nor `keep` is given: the C call itself allocates nothing);
    `keep` [n_layers, 2, n, d] receives every layer's input and output."""
    L = len(handles)
    arr = (ctypes.c_void_p * L)(*handles)
    ga = (ctypes.c_void_p * L)(*[_ptr(g) for g in gammas]) if gammas is not None else None
    be = (ctypes.c_void_p * L)(*[_ptr(b) for b in betas]) if betas is not None else None
    desc = StackDesc(L, arr, 1 if normalise else 0, ga, be, eps, 1 if residual else 0)
    n = x.shape[0]
    if work is None and keep is None:
        work = torch.empty(2, *x.shape, dtype=x.dtype, device=x.device)
    wb = work.numel() * work.element_size() if work is not None else 0
    kb = keep.numel() * keep.element_size() if keep is not None else 0
    _check(load_library().tardis_stack_forward(ctypes.byref(desc), _ptr(x), _ptr(y), _ptr(work), wb, _ptr(keep), kb, n,
                                               _stream(stream)), "tardis_stack_forward")


def tardis_debug_damage_guard(handle: int, front: bool, repair: bool):
    """Changes (or restores) four guard bytes next to the handle's fp32 accumulator; tardis_stats then reports CORRUPT."""
    _check(load_library().tardis_debug_damage_guard(handle, 1 if front else 0, 1 if repair else 0), "tardis_debug_damage_guard")


def tardis_debug_live_allocations():
    """(count, bytes) of the library's live device allocations in this process."""
    c, b = ctypes.c_int64(), ctypes.c_int64()
    _check(load_library().tardis_debug_live_allocations(ctypes.byref(c), ctypes.byref(b)), "tardis_debug_live_allocations")
    return c.value, b.value


def tardis_debug_fail_alloc(nth: int):
    """The library's (nth + 1)-th device allocation from now fails once; nth < 0 switches the injection off."""
    _check(load_library().tardis_debug_fail_alloc(nth), "tardis_debug_fail_alloc")


def tardis_save(handle: int, path: str):
    """Writes the handle's state (folded matrix, predictor, original weights, tables) to a binary file."""
    _check(load_library().tardis_save(handle, os.fsencode(path)), "tardis_save")


def tardis_load(path: str, stream=None) -> int:
    """Reads a file written by tardis_save and returns a new handle on the current device."""
    out = ctypes.c_void_p()
    _check(load_library().tardis_load(os.fsencode(path), _stream(stream), ctypes.byref(out)), "tardis_load")
    return out.value


def tardis_destroy(handle: int):
    _check(load_library().tardis_destroy(handle), "tardis_destroy")


def fold_layer(layer, stream=None, flags=0) -> int:
    """Convenience: tardis_fold from an object with the fields W1, W2, b1, b2, lo, hi, a, c, codes, scale,
    zero and cfg.group / cfg.act / cfg.bits (all CUDA tensors)."""
    return tardis_fold(layer.W1, layer.W2, layer.lo, layer.hi, layer.a, layer.c, layer.codes, layer.scale,
                       layer.zero, layer.cfg.group, b1=layer.b1, b2=layer.b2, act=layer.cfg.act,
                       pred_bits=layer.cfg.bits, stream=stream, flags=flags)
