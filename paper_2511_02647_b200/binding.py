"""ctypes binding of include/fedattn.h.  Function names match the C entry points; torch tensors
supply device memory and the current CUDA stream."""
from __future__ import annotations

import ctypes as C
import importlib.machinery
import importlib.util
import os
import warnings
from typing import Optional, Sequence

import torch

from .build import marshal_path

_PKG = os.path.dirname(os.path.abspath(__file__))
# FEDATTN_LIBRARY overrides the path of the shared library (e.g. an instrumented build).
_LIB_PATH = os.environ.get("FEDATTN_LIBRARY") or os.path.join(_PKG, "lib", "libfedattn.so")

F32, BF16 = 0, 1
AGG_CONCAT, AGG_TOPK_KNORM, AGG_INDEXED, AGG_TOPK_TOKEN = 0, 1, 2, 3
DECODE_LOCAL, DECODE_SYNC = 0, 1

_SYMBOLS = ["fedattn_workspace_bytes", "fedattn_create", "fedattn_destroy", "fedattn_status_string",
            "fedattn_poll", "fedattn_launch_count", "fedattn_tensor_core_launch_count",
            "fedattn_selftest_wait_timeout", "fedattn_local", "fedattn_aggregate_kv",
            "fedattn_sync", "fedattn_sync_remote", "fedattn_merge", "fedattn_decode", "fedattn_decode_noalloc",
            "fedattn_qk_norm_rope", "fedattn_quantize_kv", "fedattn_dequantize_kv", "fedattn_decode_quant",
            "fedattn_local_window", "fedattn_decode_window"]


class FedAttnError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__("%s failed: %s (status %d)" % (where, status_string(code), code))


class Shape(C.Structure):
    """Mirror of fedattn_shape."""
    _fields_ = [("n_participants", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("dtype", C.c_int32), ("causal", C.c_int32), ("scale", C.c_float)]

    def __init__(self, n_participants, n_q_heads, n_kv_heads, head_dim, dtype, causal=1, scale=0.0):
        super().__init__(int(n_participants), int(n_q_heads), int(n_kv_heads), int(head_dim), int(dtype),
                         int(causal), float(scale))

    @property
    def torch_dtype(self):
        return torch.bfloat16 if self.dtype == BF16 else torch.float32


def library_path() -> str:
    return _LIB_PATH


class _AllThroughCtypes:
    """What stands for the marshalling module where there is none: it takes nothing."""

    @staticmethod
    def pointer(_):
        return None

    pointers = int32s = pointer


def _load_marshal():
    """The native marshalling module (csrc/marshal.cpp).  It only saves host time: without one for this torch and this
    interpreter (a library from elsewhere, a tree built earlier, no Python headers) the same calls go through ctypes."""
    name, path = "_fedattn_marshal", marshal_path()
    try:
        loader = importlib.machinery.ExtensionFileLoader(name, path)
        module = importlib.util.module_from_spec(importlib.util.spec_from_loader(name, loader))
        loader.exec_module(module)
        return module
    except ImportError as e:
        warnings.warn("FedAttn marshalling module not loaded (%s): arguments go through ctypes, 10 us more for an "
                      "aggregation of 16 participants; `python paper_2511_02647_b200/build.py` builds it" % e, RuntimeWarning)
        return _AllThroughCtypes


def _load():
    if not os.path.exists(_LIB_PATH):
        raise ImportError("FedAttn CUDA library missing: %s (run `python paper_2511_02647_b200/build.py` "
                          "or __graft_entry__.build()); there is no fallback path" % _LIB_PATH)
    lib = C.CDLL(_LIB_PATH)
    vp, i32, i64 = C.c_void_p, C.c_int32, C.c_int64
    lib.fedattn_workspace_bytes.restype = C.c_size_t
    lib.fedattn_workspace_bytes.argtypes = [C.POINTER(Shape), i64, i64]
    lib.fedattn_create.restype = C.c_int
    lib.fedattn_create.argtypes = [C.POINTER(vp), C.c_int, vp, C.c_size_t]
    lib.fedattn_destroy.restype = None
    lib.fedattn_destroy.argtypes = [vp]
    lib.fedattn_status_string.restype = C.c_char_p
    lib.fedattn_status_string.argtypes = [C.c_int]
    lib.fedattn_poll.restype = C.c_int
    lib.fedattn_poll.argtypes = [vp, vp]
    lib.fedattn_launch_count.restype = i64
    lib.fedattn_launch_count.argtypes = [vp]
    lib.fedattn_tensor_core_launch_count.restype = i64
    lib.fedattn_tensor_core_launch_count.argtypes = [vp]
    lib.fedattn_selftest_wait_timeout.restype = C.c_int
    lib.fedattn_selftest_wait_timeout.argtypes = [vp, i32, vp]
    lib.fedattn_local.restype = C.c_int
    lib.fedattn_local.argtypes = [vp, C.POINTER(Shape), vp, vp, vp, vp, vp, vp, vp]
    lib.fedattn_aggregate_kv.restype = C.c_int
    lib.fedattn_aggregate_kv.argtypes = [vp, C.POINTER(Shape), i32, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.fedattn_sync.restype = C.c_int
    lib.fedattn_sync.argtypes = [vp, C.POINTER(Shape), vp, i64, vp, vp, vp, vp, i64, i32, vp, vp, vp]
    lib.fedattn_sync_remote.restype = C.c_int
    lib.fedattn_sync_remote.argtypes = [vp, C.POINTER(Shape), vp, vp, vp, vp, vp, i64, i32, vp, vp, vp]
    lib.fedattn_merge.restype = C.c_int
    lib.fedattn_merge.argtypes = [vp, C.POINTER(Shape), i64, vp, vp, vp, vp, vp, vp, vp]
    lib.fedattn_decode.restype = C.c_int
    lib.fedattn_decode.argtypes = [vp, C.POINTER(Shape), i32, vp, vp, vp, i64, vp, i32, vp, vp, vp]
    lib.fedattn_decode_noalloc.restype = C.c_int
    lib.fedattn_decode_noalloc.argtypes = [C.POINTER(Shape), i32, vp, vp, vp, i64, vp, i32, vp, vp, vp]
    lib.fedattn_local_window.restype = C.c_int
    lib.fedattn_local_window.argtypes = [vp, C.POINTER(Shape), vp, vp, vp, vp, i32, i32, vp, vp, vp]
    lib.fedattn_decode_window.restype = C.c_int
    lib.fedattn_decode_window.argtypes = [vp, C.POINTER(Shape), i32, vp, vp, vp, i64, vp, i32, i32, i32, vp, vp, vp]
    lib.fedattn_qk_norm_rope.restype = C.c_int
    lib.fedattn_qk_norm_rope.argtypes = [vp, C.POINTER(Shape), i64, vp, i64, vp, i64, vp, vp, C.c_float, vp, vp, i32, i32, vp,
                                         vp, vp]
    lib.fedattn_quantize_kv.restype = C.c_int
    lib.fedattn_quantize_kv.argtypes = [vp, C.POINTER(Shape), i64, vp, i64, vp, i64, vp, i64, i64, vp, vp, vp, vp, vp]
    lib.fedattn_dequantize_kv.restype = C.c_int
    lib.fedattn_dequantize_kv.argtypes = [vp, C.POINTER(Shape), i64, vp, i64, i64, vp, vp, vp, vp, vp, vp, vp]
    lib.fedattn_decode_quant.restype = C.c_int
    lib.fedattn_decode_quant.argtypes = [vp, C.POINTER(Shape), i32, vp, vp, vp, vp, vp, i64, vp, i32, i32, i32, vp, vp, vp]
    return lib


_lib = _load()
_marshal = _load_marshal()


def exported_symbols():
    """Names declared in include/fedattn.h that the loaded library exports."""
    return [s for s in _SYMBOLS if hasattr(_lib, s)]


def status_string(code: int) -> str:
    return _lib.fedattn_status_string(int(code)).decode()


def _check(code: int, where: str):
    if code != 0:
        raise FedAttnError(code, where)


# Arrays travel as bytes objects that hold the C array (parameters declared void *), which the argument tuple keeps
# alive; what the native module does not take (it answers None) goes through ctypes below.
def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    p = _marshal.pointer(t)
    if p is not None:
        return p
    if not t.is_contiguous():
        raise ValueError("tensor must be contiguous")
    return t.data_ptr()


def _ptr_array(ts):
    """Pointers of a list of tensors (or None)."""
    packed = _marshal.pointers(ts)
    return packed if packed is not None else (C.c_void_p * len(ts))(*[_ptr(t) for t in ts])


# The current stream as an integer.  torch.cuda.current_stream() builds a Stream object first: 3.2 us of the 5.3 us
# that marshalling a call took, against 0.3 us, where the whole C call takes 5.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_current_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream) -> int:
    if stream is None:
        if _raw_stream is not None and _current_device is not None and torch.cuda.is_initialized():
            return _raw_stream(_current_device())
        return torch.cuda.current_stream().cuda_stream
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _i32_array(xs: Sequence[int]):
    packed = _marshal.int32s(xs)
    return packed if packed is not None else (C.c_int32 * len(xs))(*[int(x) for x in xs])


def fedattn_workspace_bytes(shape: Shape, max_total_tokens: int, max_total_kv: int) -> int:
    return int(_lib.fedattn_workspace_bytes(C.byref(shape), int(max_total_tokens), int(max_total_kv)))


class Context:
    """Owns a device workspace tensor and the library context built around it."""

    def __init__(self, shape: Shape, max_total_tokens: int, max_total_kv: int, device: int = 0):
        nbytes = fedattn_workspace_bytes(shape, max_total_tokens, max_total_kv)
        if nbytes == 0:
            raise FedAttnError(1, "fedattn_workspace_bytes")
        self.device = int(device)
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device="cuda:%d" % self.device)
        self._h = C.c_void_p()
        _check(_lib.fedattn_create(C.byref(self._h), self.device, self.workspace.data_ptr(), nbytes),
               "fedattn_create")

    @property
    def handle(self):
        return self._h

    def poll(self, stream=None) -> int:
        """Synchronise the stream and return (and clear) the device status word."""
        return int(_lib.fedattn_poll(self._h, _stream(stream)))

    def launch_count(self) -> int:
        return int(_lib.fedattn_launch_count(self._h))

    def tensor_core_launch_count(self) -> int:
        return int(_lib.fedattn_tensor_core_launch_count(self._h))

    def selftest_wait_timeout(self, max_polls: int = 64, stream=None):
        """Launches the kernel whose bounded wait runs out (raises the TIMEOUT status word)."""
        _check(_lib.fedattn_selftest_wait_timeout(self._h, int(max_polls), _stream(stream)),
               "fedattn_selftest_wait_timeout")

    def close(self):
        if self._h:
            _lib.fedattn_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# Every entry point comes in two forms: ``fedattn_x(...)`` marshals its arguments and calls the library;
# ``prepare_x(...)`` marshals once and returns a zero-argument callable that repeats the same call (same
# buffers, same stream), for loops in which the per-call marshalling of tensors and pointer arrays would
# cost more host time than the kernel takes on the device.  Both do argument marshalling only.
class PreparedCall:
    """A library call with its arguments already converted; calling it enqueues the work again."""

    def __init__(self, fn, args, where: str, keep):
        # Numbers become C objects of their parameter's type here, once, and the function pointer of the call declares no types:
        # ctypes then passes everything as it is (17 arguments: 4.2 -> 2.5 us where a refused call was timed).
        args = tuple(t(a) if isinstance(a, (int, float)) else a for t, a in zip(fn.argtypes, args))
        self._fn, self._args, self._where, self._keep = _lib[where], args, where, keep      # (every _lib[name] is a new function object)
        self._fn.restype = C.c_int

    def __call__(self, stream=None):
        # every entry point takes the stream last; `stream` (a raw cudaStream_t as an int or a c_void_p, or an object that has one as
        # its ctypes parameter, as torch's streams do) replaces the prepared one
        if stream is None:
            code = self._fn(*self._args)
        else:
            stream = getattr(stream, "_as_parameter_", stream)
            code = self._fn(*self._args[:-1], stream if isinstance(stream, C.c_void_p) else C.c_void_p(stream))
        if code != 0:
            raise FedAttnError(code, self._where)


def _args_local(ctx, shape, q, k, v, cu_seqlens_host, o, lse, stream):
    if len(cu_seqlens_host) != shape.n_participants + 1:
        raise ValueError("cu_seqlens must have N+1 entries")
    cu = _i32_array(cu_seqlens_host)
    return (ctx.handle, C.byref(shape), _ptr(q), _ptr(k), _ptr(v), cu, _ptr(o), _ptr(lse), _stream(stream))


def fedattn_local(ctx: Context, shape: Shape, q, k, v, cu_seqlens_host: Sequence[int], o, lse=None,
                  stream=None):
    _check(_lib.fedattn_local(*_args_local(ctx, shape, q, k, v, cu_seqlens_host, o, lse, stream)), "fedattn_local")


def prepare_local(ctx: Context, shape: Shape, q, k, v, cu_seqlens_host: Sequence[int], o, lse=None, stream=None):
    return PreparedCall(_lib.fedattn_local, _args_local(ctx, shape, q, k, v, cu_seqlens_host, o, lse, stream),
                        "fedattn_local", (ctx, shape, q, k, v, o, lse))


def _args_aggregate_kv(ctx, shape, mode, k_parts, v_parts, seqlens_host, k_sel_host, sel_idx_in, k_agg, v_agg, kv_pos,
                       cu_kv, sel_idx_out, stream):
    n = shape.n_participants
    if len(k_parts) != n or len(v_parts) != n or len(seqlens_host) != n:
        raise ValueError("need one K part, V part and length per participant")
    kp, vp = _ptr_array(k_parts), _ptr_array(v_parts)
    ks = None if k_sel_host is None else _i32_array(k_sel_host)
    return (ctx.handle, C.byref(shape), int(mode), kp, vp, _i32_array(seqlens_host), ks, _ptr(sel_idx_in), _ptr(k_agg),
            _ptr(v_agg), _ptr(kv_pos), _ptr(cu_kv), _ptr(sel_idx_out), _stream(stream))


def fedattn_aggregate_kv(ctx: Context, shape: Shape, mode: int, k_parts, v_parts, seqlens_host,
                         k_sel_host=None, sel_idx_in=None, k_agg=None, v_agg=None, kv_pos=None, cu_kv=None,
                         sel_idx_out=None, stream=None):
    _check(_lib.fedattn_aggregate_kv(*_args_aggregate_kv(ctx, shape, mode, k_parts, v_parts, seqlens_host, k_sel_host,
                                                         sel_idx_in, k_agg, v_agg, kv_pos, cu_kv, sel_idx_out, stream)),
           "fedattn_aggregate_kv")


def prepare_aggregate_kv(ctx: Context, shape: Shape, mode: int, k_parts, v_parts, seqlens_host, k_sel_host=None,
                         sel_idx_in=None, k_agg=None, v_agg=None, kv_pos=None, cu_kv=None, sel_idx_out=None, stream=None):
    return PreparedCall(_lib.fedattn_aggregate_kv,
                        _args_aggregate_kv(ctx, shape, mode, k_parts, v_parts, seqlens_host, k_sel_host, sel_idx_in, k_agg,
                                           v_agg, kv_pos, cu_kv, sel_idx_out, stream),
                        "fedattn_aggregate_kv", (ctx, shape, list(k_parts), list(v_parts), sel_idx_in, k_agg, v_agg, kv_pos,
                                                 cu_kv, sel_idx_out))


def _args_sync(ctx, shape, q, q_pos, k_agg, v_agg, kv_pos, total_kv, kv_head_major, o, lse, stream):
    return (ctx.handle, C.byref(shape), _ptr(q), int(q.shape[0]), _ptr(q_pos), _ptr(k_agg), _ptr(v_agg), _ptr(kv_pos),
            int(total_kv), int(bool(kv_head_major)), _ptr(o), _ptr(lse), _stream(stream))


def fedattn_sync(ctx: Context, shape: Shape, q, q_pos, k_agg, v_agg, kv_pos, total_kv: int,
                 kv_head_major: bool, o, lse=None, stream=None):
    _check(_lib.fedattn_sync(*_args_sync(ctx, shape, q, q_pos, k_agg, v_agg, kv_pos, total_kv, kv_head_major, o, lse,
                                         stream)), "fedattn_sync")


def prepare_sync(ctx: Context, shape: Shape, q, q_pos, k_agg, v_agg, kv_pos, total_kv: int, kv_head_major: bool, o,
                 lse=None, stream=None):
    return PreparedCall(_lib.fedattn_sync,
                        _args_sync(ctx, shape, q, q_pos, k_agg, v_agg, kv_pos, total_kv, kv_head_major, o, lse, stream),
                        "fedattn_sync", (ctx, shape, q, q_pos, k_agg, v_agg, kv_pos, o, lse))


def _args_sync_remote(ctx, shape, q, cu_seqlens_host, k_agg, v_agg, kv_pos, total_kv, kv_head_major, o, lse, stream):
    if len(cu_seqlens_host) != shape.n_participants + 1:
        raise ValueError("cu_seqlens must have N+1 entries")
    cu = _i32_array(cu_seqlens_host)
    return (ctx.handle, C.byref(shape), _ptr(q), cu, _ptr(k_agg), _ptr(v_agg), _ptr(kv_pos), int(total_kv),
            int(bool(kv_head_major)), _ptr(o), _ptr(lse), _stream(stream))


def fedattn_sync_remote(ctx: Context, shape: Shape, q, cu_seqlens_host: Sequence[int], k_agg, v_agg, kv_pos,
                        total_kv: int, kv_head_major: bool, o, lse, stream=None):
    _check(_lib.fedattn_sync_remote(*_args_sync_remote(ctx, shape, q, cu_seqlens_host, k_agg, v_agg, kv_pos, total_kv,
                                                       kv_head_major, o, lse, stream)), "fedattn_sync_remote")


def prepare_sync_remote(ctx: Context, shape: Shape, q, cu_seqlens_host: Sequence[int], k_agg, v_agg, kv_pos, total_kv: int,
                        kv_head_major: bool, o, lse, stream=None):
    return PreparedCall(_lib.fedattn_sync_remote,
                        _args_sync_remote(ctx, shape, q, cu_seqlens_host, k_agg, v_agg, kv_pos, total_kv, kv_head_major, o,
                                          lse, stream),
                        "fedattn_sync_remote", (ctx, shape, q, k_agg, v_agg, kv_pos, o, lse))


def _args_merge(ctx, shape, n_rows, o_a, lse_a, o_b, lse_b, o, lse, stream):
    return (ctx.handle, C.byref(shape), int(n_rows), _ptr(o_a), _ptr(lse_a), _ptr(o_b), _ptr(lse_b), _ptr(o), _ptr(lse),
            _stream(stream))


def fedattn_merge(ctx: Context, shape: Shape, n_rows: int, o_a, lse_a, o_b, lse_b, o, lse=None, stream=None):
    _check(_lib.fedattn_merge(*_args_merge(ctx, shape, n_rows, o_a, lse_a, o_b, lse_b, o, lse, stream)), "fedattn_merge")


def prepare_merge(ctx: Context, shape: Shape, n_rows: int, o_a, lse_a, o_b, lse_b, o, lse=None, stream=None):
    return PreparedCall(_lib.fedattn_merge, _args_merge(ctx, shape, n_rows, o_a, lse_a, o_b, lse_b, o, lse, stream),
                        "fedattn_merge", (ctx, shape, o_a, lse_a, o_b, lse_b, o, lse))


def _args_decode(ctx, shape, mode, q, k_cache, v_cache, cache_stride_participant, kv_len, max_kv_len, o, lse, stream):
    return (ctx.handle, C.byref(shape), int(mode), _ptr(q), _ptr(k_cache), _ptr(v_cache), int(cache_stride_participant),
            _ptr(kv_len), int(max_kv_len), _ptr(o), _ptr(lse), _stream(stream))


def fedattn_decode(ctx: Context, shape: Shape, mode: int, q, k_cache, v_cache, cache_stride_participant: int,
                   kv_len, max_kv_len: int, o, lse=None, stream=None):
    _check(_lib.fedattn_decode(*_args_decode(ctx, shape, mode, q, k_cache, v_cache, cache_stride_participant, kv_len,
                                             max_kv_len, o, lse, stream)), "fedattn_decode")


def prepare_decode(ctx: Context, shape: Shape, mode: int, q, k_cache, v_cache, cache_stride_participant: int, kv_len,
                   max_kv_len: int, o, lse=None, stream=None):
    return PreparedCall(_lib.fedattn_decode,
                        _args_decode(ctx, shape, mode, q, k_cache, v_cache, cache_stride_participant, kv_len, max_kv_len, o,
                                     lse, stream),
                        "fedattn_decode", (ctx, shape, q, k_cache, v_cache, kv_len, o, lse))


def fedattn_decode_noalloc(shape: Shape, mode: int, q, k_cache, v_cache, cache_stride_participant: int,
                           kv_len, max_kv_len: int, o, lse=None, stream=None):
    """fedattn_decode for callers that may not allocate: no context, no workspace; the split-KV
    partials use a fixed array inside the library (bf16, head_dim 128, at most 256 output rows).
    Runs on the current CUDA device; calls that may overlap on the GPU share that array and race."""
    _check(_lib.fedattn_decode_noalloc(C.byref(shape), int(mode), _ptr(q), _ptr(k_cache), _ptr(v_cache),
                                       int(cache_stride_participant), _ptr(kv_len), int(max_kv_len), _ptr(o),
                                       _ptr(lse), _stream(stream)), "fedattn_decode_noalloc")


# ---- windows, queries and keys before attention, and the 4-bit cache ---------------------------------------------------
# These calls take tensors of several kinds; what the C call cannot see (types, shapes, strides) is checked here.
def _stream_of(ctx: Context, stream) -> int:
    """The current stream of the context's device, which need not be the current device."""
    if stream is None and _raw_stream is not None and torch.cuda.is_initialized():
        return _raw_stream(ctx.device)
    return torch.cuda.current_stream(ctx.device).cuda_stream if stream is None else _stream(stream)


def _i32(x) -> int:
    """A number as an int32 parameter takes it, which would drop what lies above its 32 bits: beyond either end it is that end, as a count
    more than any length, and where that is no valid value the C call refuses it."""
    return max(-2 ** 31, min(int(x), 2 ** 31 - 1))


def _tensor(ctx: Context, t, dtype, shape, what: str):
    """Pointer of a contiguous tensor of this type and shape on the context's device; None stays None."""
    if t is None:
        return None
    if t.dtype != dtype or tuple(t.shape) != tuple(shape):
        raise ValueError("%s must be %s of shape %s, not %s of shape %s" % (what, dtype, tuple(shape), t.dtype, tuple(t.shape)))
    if t.device.index != ctx.device:
        raise ValueError("%s must be on device %d" % (what, ctx.device))
    return _ptr(t)


def _rows(ctx: Context, t, n_rows: int, heads: int, shape: Shape, what: str):
    """Pointer and row stride (in elements, 0 for packed) of [n_rows, heads, head_dim] whose rows are contiguous."""
    if t is None:
        return None, 0
    d = shape.head_dim
    if t.dtype != shape.torch_dtype or tuple(t.shape) != (n_rows, heads, d):
        raise ValueError("%s must be %s of shape %s, not %s of shape %s" % (what, shape.torch_dtype, (n_rows, heads, d), t.dtype,
                                                                             tuple(t.shape)))
    if t.device.index != ctx.device:
        raise ValueError("%s must be on device %d" % (what, ctx.device))
    if t.stride(2) != 1 or (heads > 1 and t.stride(1) != d) or (n_rows > 1 and t.stride(0) < heads * d):
        raise ValueError("%s: the heads of a row must be contiguous, and rows must not overlap" % what)
    return t.data_ptr(), t.stride(0) if n_rows > 1 else 0


def _args_local_window(ctx, shape, q, k, v, cu_seqlens_host, window, n_sink, o, lse, stream):
    if len(cu_seqlens_host) != shape.n_participants + 1:
        raise ValueError("cu_seqlens must have N+1 entries")
    if not 0 <= min(cu_seqlens_host) <= max(cu_seqlens_host) < 2 ** 31:
        raise ValueError("cu_seqlens must be within 0 .. 2^31 - 1")
    L, hq, hkv, d, dt = int(q.shape[0]), shape.n_q_heads, shape.n_kv_heads, shape.head_dim, shape.torch_dtype
    if L != cu_seqlens_host[-1]:
        raise ValueError("q has %d rows, the segments %d" % (L, cu_seqlens_host[-1]))
    return (ctx.handle, C.byref(shape), _tensor(ctx, q, dt, (L, hq, d), "q"), _tensor(ctx, k, dt, (L, hkv, d), "k"),
            _tensor(ctx, v, dt, (L, hkv, d), "v"), _i32_array(cu_seqlens_host), _i32(window), _i32(n_sink),
            _tensor(ctx, o, dt, (L, hq, d), "o"), _tensor(ctx, lse, torch.float32, (L, hq), "lse"), _stream_of(ctx, stream))


def fedattn_local_window(ctx: Context, shape: Shape, q, k, v, cu_seqlens_host: Sequence[int], window: int, n_sink: int, o,
                         lse=None, stream=None):
    """fedattn_local through a sliding window (|i - j| < window) with the segment's first n_sink rows always visible."""
    _check(_lib.fedattn_local_window(*_args_local_window(ctx, shape, q, k, v, cu_seqlens_host, window, n_sink, o, lse, stream)),
           "fedattn_local_window")


def prepare_local_window(ctx: Context, shape: Shape, q, k, v, cu_seqlens_host: Sequence[int], window: int, n_sink: int, o,
                         lse=None, stream=None):
    return PreparedCall(_lib.fedattn_local_window,
                        _args_local_window(ctx, shape, q, k, v, cu_seqlens_host, window, n_sink, o, lse, stream),
                        "fedattn_local_window", (ctx, shape, q, k, v, o, lse))


def _args_decode_window(ctx, shape, mode, q, k_cache, v_cache, cache_stride_participant, kv_len, max_kv_len, window, n_sink, o,
                        lse, stream):
    n, dt = shape.n_participants, shape.torch_dtype
    rows = (n, shape.n_q_heads, shape.head_dim)
    row = shape.n_kv_heads * shape.head_dim
    held = int(max_kv_len) * row + (0 if int(mode) == DECODE_SYNC else (n - 1) * int(cache_stride_participant))
    if min(k_cache.numel(), v_cache.numel()) < held:
        raise ValueError("the caches have %d and %d elements, the call may read %d" % (k_cache.numel(), v_cache.numel(), held))
    return (ctx.handle, C.byref(shape), _i32(mode), _tensor(ctx, q, dt, rows, "q"),
            *[_tensor(ctx, t, dt, t.shape, "cache") for t in (k_cache, v_cache)], int(cache_stride_participant),
            _tensor(ctx, kv_len, torch.int32, (1 if int(mode) == DECODE_SYNC else n,), "kv_len"), _i32(max_kv_len), _i32(window),
            _i32(n_sink), _tensor(ctx, o, dt, rows, "o"), _tensor(ctx, lse, torch.float32, rows[:2], "lse"),
            _stream_of(ctx, stream))


def fedattn_decode_window(ctx: Context, shape: Shape, mode: int, q, k_cache, v_cache, cache_stride_participant: int, kv_len,
                          max_kv_len: int, window: int, n_sink: int, o, lse=None, stream=None):
    """fedattn_decode over the last `window` cached rows and the first n_sink."""
    _check(_lib.fedattn_decode_window(*_args_decode_window(ctx, shape, mode, q, k_cache, v_cache, cache_stride_participant, kv_len,
                                                           max_kv_len, window, n_sink, o, lse, stream)), "fedattn_decode_window")


def prepare_decode_window(ctx: Context, shape: Shape, mode: int, q, k_cache, v_cache, cache_stride_participant: int, kv_len,
                          max_kv_len: int, window: int, n_sink: int, o, lse=None, stream=None):
    return PreparedCall(_lib.fedattn_decode_window,
                        _args_decode_window(ctx, shape, mode, q, k_cache, v_cache, cache_stride_participant, kv_len, max_kv_len,
                                            window, n_sink, o, lse, stream),
                        "fedattn_decode_window", (ctx, shape, q, k_cache, v_cache, kv_len, o, lse))


def _args_qk_norm_rope(ctx, shape, q, k, q_weight, k_weight, eps, pos, inv_freq, interleaved, q_out, k_out, stream):
    if q is None and k is None:
        raise ValueError("need q or k")
    n = int((q if q is not None else k).shape[0])
    hq, hkv, d, dt = shape.n_q_heads, shape.n_kv_heads, shape.head_dim, shape.torch_dtype
    qp, qs = _rows(ctx, q, n, hq, shape, "q")
    kp, ks = _rows(ctx, k, n, hkv, shape, "k")
    freq = None if inv_freq is None or len(inv_freq) == 0 else (C.c_double * len(inv_freq))(*[float(x) for x in inv_freq])
    return (ctx.handle, C.byref(shape), n, qp, qs, kp, ks, _tensor(ctx, q_weight, dt, (d,), "q_weight"),
            _tensor(ctx, k_weight, dt, (d,), "k_weight"), float(eps), _tensor(ctx, pos, torch.int32, (n,), "pos"), freq,
            2 * len(freq) if freq is not None else 0, int(bool(interleaved)), _tensor(ctx, q_out, dt, (n, hq, d), "q_out"),
            _tensor(ctx, k_out, dt, (n, hkv, d), "k_out"), _stream_of(ctx, stream))


def fedattn_qk_norm_rope(ctx: Context, shape: Shape, q, k, q_weight, k_weight, eps: float, pos, inv_freq: Sequence[float],
                         interleaved: bool, q_out, k_out, stream=None):
    """RMS norm per head of queries and keys, then the rotation by position.  q [n, Hq, d] and k [n, Hkv, d] may be strided
    over rows (slices of joint projections); inv_freq: rot_dim / 2 host numbers, radians per position."""
    _check(_lib.fedattn_qk_norm_rope(*_args_qk_norm_rope(ctx, shape, q, k, q_weight, k_weight, eps, pos, inv_freq, interleaved,
                                                         q_out, k_out, stream)), "fedattn_qk_norm_rope")


def prepare_qk_norm_rope(ctx: Context, shape: Shape, q, k, q_weight, k_weight, eps: float, pos, inv_freq: Sequence[float],
                         interleaved: bool, q_out, k_out, stream=None):
    return PreparedCall(_lib.fedattn_qk_norm_rope,
                        _args_qk_norm_rope(ctx, shape, q, k, q_weight, k_weight, eps, pos, inv_freq, interleaved, q_out, k_out,
                                           stream),
                        "fedattn_qk_norm_rope", (ctx, shape, q, k, q_weight, k_weight, pos, q_out, k_out))


class QuantCache:
    """The four device arrays of 4-bit caches: codes uint8 [n_caches, Hkv, cap_rows, d/2], scales uint8
    [n_caches, Hkv, cap_rows, d/32], for keys and for values.  cap_rows: multiple of 16.  Arrays that are not given are
    allocated, zeroed."""

    def __init__(self, shape: Shape, n_caches: int, cap_rows: int, k_codes=None, k_scales=None, v_codes=None, v_scales=None,
                 device: int = 0):
        self.n_caches, self.cap_rows = int(n_caches), int(cap_rows)
        if shape.head_dim % 32 or self.cap_rows % 16 or self.cap_rows < 0 or self.n_caches < 1:
            raise ValueError("4-bit caches need head_dim a multiple of 32 and cap_rows a multiple of 16")
        rows = (self.n_caches, shape.n_kv_heads, self.cap_rows)
        given = {"k_codes": k_codes, "k_scales": k_scales, "v_codes": v_codes, "v_scales": v_scales}
        for name, t in given.items():
            want = rows + (shape.head_dim // (2 if name.endswith("codes") else 32),)
            if t is None:
                t = torch.zeros(want, dtype=torch.uint8, device="cuda:%d" % device)
            if t.dtype != torch.uint8 or tuple(t.shape) != want or not t.is_contiguous() or t.device.type != "cuda":
                raise ValueError("%s must be contiguous uint8 of shape %s on a GPU" % (name, want))
            setattr(self, name, t)

    def arrays(self):
        return self.k_codes, self.k_scales, self.v_codes, self.v_scales


def _cache(ctx, shape, cache: QuantCache):
    rows = (cache.n_caches, shape.n_kv_heads, cache.cap_rows)
    return [_tensor(ctx, t, torch.uint8, rows + (w,), "cache") for t, w in
            zip(cache.arrays(), (shape.head_dim // 2, shape.head_dim // 32) * 2)]


def _args_quantize_kv(ctx, shape, k, v, at, cache, stream):
    n = int(k.shape[0])
    kp, ks = _rows(ctx, k, n, shape.n_kv_heads, shape, "k")
    vp, vs = _rows(ctx, v, n, shape.n_kv_heads, shape, "v")
    return (ctx.handle, C.byref(shape), n, kp, ks, vp, vs, _tensor(ctx, at, torch.int32, (n,), "at"), cache.n_caches,
            cache.cap_rows, *_cache(ctx, shape, cache), _stream_of(ctx, stream))


def fedattn_quantize_kv(ctx: Context, shape: Shape, k, v, at, cache: QuantCache, stream=None):
    """Rows of k, v [n, Hkv, d] (strided over rows or packed) into 4-bit caches: row i to flat row at[i] (int32, distinct;
    negative: skipped; None: i)."""
    _check(_lib.fedattn_quantize_kv(*_args_quantize_kv(ctx, shape, k, v, at, cache, stream)), "fedattn_quantize_kv")


def prepare_quantize_kv(ctx: Context, shape: Shape, k, v, at, cache: QuantCache, stream=None):
    return PreparedCall(_lib.fedattn_quantize_kv, _args_quantize_kv(ctx, shape, k, v, at, cache, stream), "fedattn_quantize_kv",
                        (ctx, shape, k, v, at, *cache.arrays()))


def _args_dequantize_kv(ctx, shape, cache, at, k, v, stream):
    n, dt = int(k.shape[0]), shape.torch_dtype
    rows = (n, shape.n_kv_heads, shape.head_dim)
    return (ctx.handle, C.byref(shape), n, _tensor(ctx, at, torch.int32, (n,), "at"), cache.n_caches, cache.cap_rows,
            *_cache(ctx, shape, cache), _tensor(ctx, k, dt, rows, "k"), _tensor(ctx, v, dt, rows, "v"), _stream_of(ctx, stream))


def fedattn_dequantize_kv(ctx: Context, shape: Shape, cache: QuantCache, at, k, v, stream=None):
    """The values of flat rows at[i] of 4-bit caches (None: rows 0, 1, ...) to rows i of k, v [n, Hkv, d]."""
    _check(_lib.fedattn_dequantize_kv(*_args_dequantize_kv(ctx, shape, cache, at, k, v, stream)), "fedattn_dequantize_kv")


def prepare_dequantize_kv(ctx: Context, shape: Shape, cache: QuantCache, at, k, v, stream=None):
    return PreparedCall(_lib.fedattn_dequantize_kv, _args_dequantize_kv(ctx, shape, cache, at, k, v, stream),
                        "fedattn_dequantize_kv", (ctx, shape, *cache.arrays(), at, k, v))


def _args_decode_quant(ctx, shape, mode, q, cache, kv_len, max_kv_len, o, lse, window, n_sink, stream):
    n = shape.n_participants
    caches = 1 if int(mode) == DECODE_SYNC else n
    if cache.n_caches != caches:
        raise ValueError("need %d caches, not %d" % (caches, cache.n_caches))
    rows = (n, shape.n_q_heads, shape.head_dim)
    return (ctx.handle, C.byref(shape), _i32(mode), _tensor(ctx, q, shape.torch_dtype, rows, "q"), *_cache(ctx, shape, cache),
            cache.cap_rows, _tensor(ctx, kv_len, torch.int32, (caches,), "kv_len"), _i32(max_kv_len), _i32(window), _i32(n_sink),
            _tensor(ctx, o, shape.torch_dtype, rows, "o"), _tensor(ctx, lse, torch.float32, rows[:2], "lse"),
            _stream_of(ctx, stream))


def fedattn_decode_quant(ctx: Context, shape: Shape, mode: int, q, cache: QuantCache, kv_len, max_kv_len: int, o, lse=None,
                         window: int = 0, n_sink: int = 0, stream=None):
    """fedattn_decode over 4-bit caches; window 0: all rows, else the last `window` and the first n_sink."""
    _check(_lib.fedattn_decode_quant(*_args_decode_quant(ctx, shape, mode, q, cache, kv_len, max_kv_len, o, lse, window, n_sink,
                                                         stream)), "fedattn_decode_quant")


def prepare_decode_quant(ctx: Context, shape: Shape, mode: int, q, cache: QuantCache, kv_len, max_kv_len: int, o, lse=None,
                         window: int = 0, n_sink: int = 0, stream=None):
    return PreparedCall(_lib.fedattn_decode_quant,
                        _args_decode_quant(ctx, shape, mode, q, cache, kv_len, max_kv_len, o, lse, window, n_sink, stream),
                        "fedattn_decode_quant", (ctx, shape, q, *cache.arrays(), kv_len, o, lse))
