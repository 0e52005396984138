"""Python binding of libragged.so: the ragged (minimally padded) transformer
encoder layer for MI355X (gfx950).

This module only marshals arguments: torch tensors provide device memory and
the current HIP stream; every step of the computation runs in the library's HIP
kernels.  There is no CPU path: importing fails loudly when the library has not
been built (``python paper_2110_10221_amd/_build.py`` or
``__graft_entry__.build()``).

Function names match the C interface in include/ragged.h.
"""
from __future__ import annotations

import ctypes
import operator
import os

import torch

from ._build import built_for

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libragged.so")

RAG_OK = 0
RAG_F32, RAG_BF16 = 0, 1
RAG_ACT_NONE, RAG_ACT_GELU_ERF, RAG_ACT_GELU_TANH = 0, 1, 2
RAG_TILE = 64
RAG_HEAD_DIM = 64
RAG_LAYER_UNFUSED_ATTENTION = 1
RAG_LAYER_CAUSAL = 2
RAG_LAYER_BUILD_PLAN = 4
RAG_LAYER_EVENTS = 10
RAG_NOALLOC_SCRATCH_BYTES = 64 << 20
DATA_BITS = {1: "negative length", 2: "length > max_len", 4: "sum of lengths != total_tokens",
             8: "qkt_cap exceeded", 16: "av_cap exceeded", 32: "score buffer too small",
             64: "keys outside the cache"}
RAG_VGEMM_TILE_M, RAG_VGEMM_TILE_N = 128, 256
RAG_VGEMM_MAX_BATCH, RAG_VGEMM_MAX_DIM, RAG_VGEMM_MAX_TILES = 4096, 65536, 1 << 30
RAG_NORM_MAX_DIM = 16384
RAG_I8_MAX_K = 131056
RAG_ROTARY_HALF, RAG_ROTARY_INTERLEAVED, RAG_ROTARY_INVERSE = 0, 1, 2
RAG_ROTARY_PLAIN, RAG_ROTARY_LINEAR, RAG_ROTARY_NTK, RAG_ROTARY_YARN = 0, 1, 2, 3
RAG_ROTARY_MAX_DIM = 512
VGEMM_DATA_BITS = {1: "negative size", 2: "size > RAG_VGEMM_MAX_DIM", 4: "tile_cap exceeded",
                   8: "operand buffer too small", 16: "bf16 needs k % 64 == 0 and n % 8 == 0"}

if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is missing: build the HIP library first "
                      "(python paper_2110_10221_amd/_build.py)")

_lib = ctypes.CDLL(LIB_PATH)

_p, _i32, _i64, _f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float


class RagPlan(ctypes.Structure):
    _fields_ = [("batch", _i32), ("total_tokens", _i32), ("max_len", _i32), ("heads", _i32),
                ("qkt_cap", _i64), ("av_cap", _i64),
                ("lengths", _p), ("tok_off", _p), ("att_off", _p), ("order", _p), ("tok_seq", _p),
                ("qkt_item_off", _p), ("av_item_off", _p), ("qkt_items", _p), ("av_items", _p),
                ("status", _p)]


class RagVgemmPlan(ctypes.Structure):
    _fields_ = [("batch", _i32), ("tile_cap", _i64), ("dims", _p), ("a_off", _p), ("b_off", _p), ("c_off", _p),
                ("order", _p), ("tile_off", _p), ("tile_items", _p), ("status", _p)]


class RagLayerWeights(ctypes.Structure):
    _fields_ = [(n, _p) for n in ("w_qkv", "b_qkv", "w_o", "b_o", "ln1_g", "ln1_b",
                                  "w_ff1", "b_ff1", "w_ff2", "b_ff2", "ln2_g", "ln2_b")]


def _sig(name, args):
    f = getattr(_lib, name)
    f.restype = ctypes.c_int32
    f.argtypes = args
    return f


_lib.ragged_status_string.restype = ctypes.c_char_p
_lib.ragged_status_string.argtypes = [_i32]
_lib.ragged_last_error.restype = ctypes.c_char_p
_lib.ragged_last_error.argtypes = []
_c_plan_capacity = _sig("ragged_plan_capacity", [_i32, _i32, _i32, _i32, ctypes.POINTER(_i64), ctypes.POINTER(_i64)])
_c_offsets = _sig("ragged_offsets", [ctypes.POINTER(RagPlan), _p])
_c_qkt = _sig("ragged_qkt", [ctypes.POINTER(RagPlan), _p, _i32, _p, _i32, _i32, _f32, _p, _i64, _i32, _p])
_c_softmax = _sig("ragged_softmax", [ctypes.POINTER(RagPlan), _p, _p, _i64, _i32, _p])
_c_attn_v = _sig("ragged_attn_v", [ctypes.POINTER(RagPlan), _p, _i64, _p, _i32, _i32, _p, _i32, _i32, _p])
_c_attention = _sig("ragged_attention", [ctypes.POINTER(RagPlan), _p, _i32, _p, _i32, _p, _i32, _i32, _f32, _p,
                                         _i32, _i32, _p])
_c_qkt_causal = _sig("ragged_qkt_causal", list(_c_qkt.argtypes))
_c_softmax_causal = _sig("ragged_softmax_causal", list(_c_softmax.argtypes))
_c_attn_v_causal = _sig("ragged_attn_v_causal", list(_c_attn_v.argtypes))
_c_attention_causal = _sig("ragged_attention_causal", list(_c_attention.argtypes))
_c_linear = _sig("packed_linear", [_p, _i32, _p, _p, _p, _i32, _i32, _p, _i32, _i32, _i32, _i32, _i32, _p])
_c_layernorm = _sig("packed_layernorm", [_p, _i32, _p, _p, _f32, _p, _i32, _i32, _i32, _i32, _p])
_c_rmsnorm = _sig("packed_rmsnorm", [_p, _i32, _p, _i32, _p, _f32, _p, _i32, _p, _i32, _p, _i32, _p, _i32, _i32, _i32, _p])
_c_quantize_i8 = _sig("packed_quantize_i8", [_p, _i32, _p, _i32, _p, _i32, _i32, _i32, _p])
_c_linear_i8 = _sig("packed_linear_i8", [_p, _i32, _p, _p, _p, _p, _p, _i32, _i32, _p, _i32, _i32, _i32, _i32, _i32, _p])
_c_window_ws = _sig("ragged_attention_window_workspace", [ctypes.POINTER(RagPlan), _i32, _i32, _i32, _i32, _i32,
                                                          ctypes.POINTER(ctypes.c_size_t)])
_c_window = _sig("ragged_attention_window", [ctypes.POINTER(RagPlan), _p, _i32, _p, _i32, _p, _i32, _i32, _i32, _f32, _i32,
                                             _i32, _p, _i32, _p, ctypes.c_size_t, _i32, _p])
_c_window_cached = _sig("ragged_attention_window_cached", [ctypes.POINTER(RagPlan), _p, _i32, _p, _i32, _p, _i32, _i64, _p,
                                                           _p, _i32, _i32, _i32, _f32, _i32, _i32, _p, _i32, _p,
                                                           ctypes.c_size_t, _i32, _p])
_f64 = ctypes.c_double
_c_rotary_frequencies = _sig("rotary_frequencies", [_i32, _f64, _i32, _f64, _i32, _f64, _f64, _p, _p])
_c_rotary = _sig("packed_rotary", [ctypes.POINTER(RagPlan), _p, _i32, _p, _i32, _i32, _i32, _i32, _i32, _p, _f32, _p,
                                   _i32, _p])
_c_vgemm_capacity = _sig("vgemm_plan_capacity", [_i32, _i32, _i32, ctypes.POINTER(_i64)])
_c_vgemm_tile_count = _sig("vgemm_tile_count", [_i32, _p, ctypes.POINTER(_i64)])
_c_vgemm_offsets = _sig("vgemm_offsets", [ctypes.POINTER(RagVgemmPlan), _p])
_c_vgemm = _sig("ragged_vgemm", [ctypes.POINTER(RagVgemmPlan), _p, _i64, _p, _i64, _p, _i64, _i32, _p])
_c_trmm = _sig("ragged_trmm", [_p, _i32, _p, _i32, _p, _i32, _i32, _i32, _i32, _p])
_c_ws = _sig("encoder_layer_workspace", [_i32, _i32, _i32, _i32, _i32, _i32, _i32, ctypes.POINTER(ctypes.c_size_t)])
_c_layer = _sig("encoder_layer", [ctypes.POINTER(RagPlan), _p, _p, _i32, _i32, _i32, _i32, _f32, _i32, _i32,
                                  ctypes.POINTER(RagLayerWeights), _p, ctypes.c_size_t, _i32, _p, _p])
_c_layer_noalloc = _sig("encoder_layer_noalloc", [ctypes.POINTER(RagPlan), _p, _p, _i32, _i32, _i32, _i32, _f32,
                                                  _i32, _i32, ctypes.POINTER(RagLayerWeights), _i32, _p])


class RaggedError(RuntimeError):
    def __init__(self, fn, status):
        self.status = status
        msg = _lib.ragged_last_error().decode()
        super().__init__(f"{fn}: {_lib.ragged_status_string(status).decode()}: {msg}")


def _check(fn, status):
    if status != RAG_OK:
        raise RaggedError(fn, status)


def library():
    """The loaded ctypes library (for callers that want the raw C entry points)."""
    return _lib


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream):
    s = torch.cuda.current_stream() if stream is None else stream
    return ctypes.c_void_p(s.cuda_stream)


def _dtype_code(t):
    if t.dtype == torch.bfloat16:
        return RAG_BF16
    if t.dtype == torch.float32:
        return RAG_F32
    raise TypeError(f"unsupported tensor dtype {t.dtype} (bfloat16 or float32)")


def _ld(t):
    if t.dim() != 2 or t.stride(1) != 1:
        raise ValueError("expected a 2-D tensor with unit column stride")
    return t.stride(0)


def ragged_plan_capacity(batch, total_tokens, max_len, heads):
    q, a = _i64(), _i64()
    _check("ragged_plan_capacity", _c_plan_capacity(batch, total_tokens, max_len, heads, ctypes.byref(q), ctypes.byref(a)))
    return q.value, a.value


class Plan:
    """Device arrays of one batch's prelude, allocated with torch on `device`.

    `lengths` is an int32 device tensor [B]; `total_tokens` and `max_len` are
    the host-side sizes the caller promises (the device checks them)."""

    def __init__(self, lengths: torch.Tensor, total_tokens: int, max_len: int, heads: int,
                 qkt_cap: int | None = None, av_cap: int | None = None):
        if lengths.dtype != torch.int32 or lengths.dim() != 1:
            raise ValueError("lengths must be a 1-D int32 device tensor")
        if not lengths.is_contiguous():
            raise ValueError("lengths must be contiguous (the kernels read lengths[b] as dense memory)")
        if not lengths.is_cuda:
            raise ValueError("lengths must be a 1-D int32 device tensor")
        dev = lengths.device
        B = lengths.numel()
        cq, ca = ragged_plan_capacity(B, total_tokens, max_len, heads)
        qkt_cap = cq if qkt_cap is None else qkt_cap
        av_cap = ca if av_cap is None else av_cap
        i32 = dict(dtype=torch.int32, device=dev)
        self.lengths = lengths
        self.tok_off = torch.empty(B + 1, **i32)
        self.att_off = torch.empty(B + 1, dtype=torch.int64, device=dev)
        self.order = torch.empty(B, **i32)
        self.tok_seq = torch.empty(max(total_tokens, 1), **i32)
        self.qkt_item_off = torch.empty(B + 1, **i32)
        self.av_item_off = torch.empty(B + 1, **i32)
        self.qkt_items = torch.empty(max(4 * qkt_cap, 4), **i32)
        self.av_items = torch.empty(max(3 * av_cap, 3), **i32)
        self.status = torch.zeros(4, **i32)
        self.batch, self.total_tokens, self.max_len, self.heads = B, total_tokens, max_len, heads
        self.qkt_cap, self.av_cap = qkt_cap, av_cap
        self.c = RagPlan(B, total_tokens, max_len, heads, qkt_cap, av_cap,
                         lengths.data_ptr(), self.tok_off.data_ptr(), self.att_off.data_ptr(),
                         self.order.data_ptr(), self.tok_seq.data_ptr(), self.qkt_item_off.data_ptr(),
                         self.av_item_off.data_ptr(), self.qkt_items.data_ptr(), self.av_items.data_ptr(),
                         self.status.data_ptr())

    def ref(self):
        return ctypes.byref(self.c)

    def data_errors(self):
        """Decode status[0] (synchronises)."""
        f = int(self.status[0].item())
        return [msg for bit, msg in DATA_BITS.items() if f & bit]


def ragged_offsets(plan: Plan, stream=None):
    _check("ragged_offsets", _c_offsets(plan.ref(), _stream(stream)))


def ragged_qkt(plan: Plan, q, k, scores, scale, head_dim=RAG_HEAD_DIM, stream=None):
    _check("ragged_qkt", _c_qkt(plan.ref(), _ptr(q), _ld(q), _ptr(k), _ld(k), head_dim, scale, _ptr(scores),
                                scores.numel(), _dtype_code(q), _stream(stream)))


def ragged_qkt_causal(plan: Plan, q, k, scores, scale, head_dim=RAG_HEAD_DIM, stream=None):
    _check("ragged_qkt_causal", _c_qkt_causal(plan.ref(), _ptr(q), _ld(q), _ptr(k), _ld(k), head_dim, scale,
                                              _ptr(scores), scores.numel(), _dtype_code(q), _stream(stream)))


def ragged_softmax(plan: Plan, scores, probs=None, stream=None):
    probs = scores if probs is None else probs
    _check("ragged_softmax", _c_softmax(plan.ref(), _ptr(scores), _ptr(probs), min(scores.numel(), probs.numel()),
                                        _dtype_code(scores), _stream(stream)))
    return probs


def ragged_softmax_causal(plan: Plan, scores, probs=None, stream=None):
    probs = scores if probs is None else probs
    _check("ragged_softmax_causal", _c_softmax_causal(plan.ref(), _ptr(scores), _ptr(probs),
                                                      min(scores.numel(), probs.numel()), _dtype_code(scores),
                                                      _stream(stream)))
    return probs


def ragged_attn_v(plan: Plan, probs, v, out, head_dim=RAG_HEAD_DIM, stream=None):
    _check("ragged_attn_v", _c_attn_v(plan.ref(), _ptr(probs), probs.numel(), _ptr(v), _ld(v), head_dim, _ptr(out),
                                      _ld(out), _dtype_code(v), _stream(stream)))


def ragged_attn_v_causal(plan: Plan, probs, v, out, head_dim=RAG_HEAD_DIM, stream=None):
    _check("ragged_attn_v_causal", _c_attn_v_causal(plan.ref(), _ptr(probs), probs.numel(), _ptr(v), _ld(v),
                                                    head_dim, _ptr(out), _ld(out), _dtype_code(v), _stream(stream)))


def ragged_attention(plan: Plan, q, k, v, out, scale, head_dim=RAG_HEAD_DIM, stream=None):
    _check("ragged_attention", _c_attention(plan.ref(), _ptr(q), _ld(q), _ptr(k), _ld(k), _ptr(v), _ld(v), head_dim,
                                            scale, _ptr(out), _ld(out), _dtype_code(q), _stream(stream)))


def ragged_attention_causal(plan: Plan, q, k, v, out, scale, head_dim=RAG_HEAD_DIM, stream=None):
    _check("ragged_attention_causal", _c_attention_causal(plan.ref(), _ptr(q), _ld(q), _ptr(k), _ld(k), _ptr(v),
                                                          _ld(v), head_dim, scale, _ptr(out), _ld(out),
                                                          _dtype_code(q), _stream(stream)))


def packed_linear(x, w, y, bias=None, residual=None, act=RAG_ACT_NONE, stream=None):
    T, K = x.shape
    N = w.shape[0]
    ldr = _ld(residual) if residual is not None else 0
    _check("packed_linear", _c_linear(_ptr(x), _ld(x), _ptr(w), _ptr(bias), _ptr(residual), ldr, act, _ptr(y), _ld(y),
                                      T, K, N, _dtype_code(x), _stream(stream)))


def packed_layernorm(x, gamma, beta, y, eps=1e-5, stream=None):
    T, d = x.shape
    _check("packed_layernorm", _c_layernorm(_ptr(x), _ld(x), _ptr(gamma), _ptr(beta), eps, _ptr(y), _ld(y), T, d,
                                            _dtype_code(x), _stream(stream)))


# The operators below check types, shapes and devices of what they are given.  A step of single tokens
# takes as long as its host side, so calls whose arguments are as documented are read, checked and
# made by _binding.so (packed_rmsnorm of 8 x 1024, call after call: 3.5 us, 6.4 by way of ctypes); it returns None, and
# launches nothing, for any other call, which then meets the checks written out here.  It is linked against
# torch: where it is missing, does not load or was built for another torch or Python, every call goes by way of ctypes.


class _Unbound:
    def __getattr__(self, name):
        return lambda *args: None


def _load_fast():
    try:
        from . import _binding
    except ImportError:
        return _Unbound()
    return _binding if getattr(_binding, "built_for", None) == built_for() else _Unbound()


_fast = _load_fast()
_fast.bind(torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream,
           *(ctypes.cast(f, _p).value for f in (_c_rmsnorm, _c_quantize_i8, _c_linear_i8, _c_rotary, _c_window, _c_window_cached)))

class _Codes(dict):
    def __missing__(self, dtype):
        raise TypeError(f"unsupported tensor dtype {dtype} (bfloat16 or float32)")


_CODES = _Codes({torch.float32: RAG_F32, torch.bfloat16: RAG_BF16})


def _refuse(name, t, shape, dtype, dev):
    raise ValueError(f"{name} must be {list(shape)} of {dtype} on device {dev} with unit stride in its last dimension, "
                     f"not {list(t.shape)} of {t.dtype} on {t.device}, strides {list(t.stride())}")


def _mat(name, t, shape, dtype, dev):
    """Leading dimension of a matrix of this shape (a tuple) and type; 0 for None."""
    if t is None:
        return 0
    ld = t.stride()
    if t.shape != shape or t.dtype is not dtype or t.get_device() != dev or ld[1] != 1 or ld[0] > 0x7fffffff:
        _refuse(name, t, shape, dtype, dev)
    return ld[0]


def _vec(name, t, n, dtype, dev):
    """Address of a contiguous vector of n elements; None for None."""
    if t is None:
        return None
    if t.shape != (n,) or t.dtype is not dtype or t.get_device() != dev or (n > 1 and t.stride()[0] != 1):
        _refuse(name, t, (n,), dtype, dev)
    return t.data_ptr()


def _addr(t):
    return None if t is None else t.data_ptr()


def _launch_stream(stream, dev, plan=None):
    """The stream to launch on: tensors (and plans) of another device than the current one are refused."""
    if dev < 0 or dev != torch.cuda.current_device() or (plan is not None and plan.status.get_device() != dev):
        raise ValueError("the tensors and the plan must be on the current device")
    # (the current stream's handle; building the Stream object takes longer than the call)
    return torch._C._cuda_getCurrentRawStream(dev) if stream is None else stream.cuda_stream


_I32_MAX = 2 ** 31 - 1


def _i32(name, n):
    """The integer itself: ctypes would wrap one past 32 bits."""
    n = operator.index(n)
    if not -_I32_MAX - 1 <= n <= _I32_MAX:
        raise ValueError(f"{name} {n} does not fit into 32 bits")
    return n


def _bound(name, n):
    """A window or a bound: past 2^31 - 1, which no position passes, the same as that."""
    return _I32_MAX if n > _I32_MAX else _i32(name, n)


def _sizes(*n):
    """The sizes themselves: ctypes would wrap larger ones."""
    if max(n) > _I32_MAX:
        raise ValueError(f"sizes {n} pass 2^31 - 1")
    return n


def packed_rmsnorm(x, gamma, y=None, eps=1e-6, residual=None, x_out=None, q=None, q_scale=None, stream=None):
    """h = x + residual, and its RMS norm times gamma: into `y`, into the 8-bit rows `q` (int8)
    and `q_scale` (float32 [T]), or both; `x_out` receives h.  `y` and `x_out` may be x or residual."""
    st = _fast.packed_rmsnorm(x, gamma, y, eps, residual, x_out, q, q_scale, stream)
    if st is None:
        st = _checked_rmsnorm(x, gamma, y, eps, residual, x_out, q, q_scale, stream)
    if st:
        _check("packed_rmsnorm", st)


def _checked_rmsnorm(x, gamma, y, eps, residual, x_out, q, q_scale, stream):
    shape, dt, dev = x.shape, x.dtype, x.get_device()
    T, d = _sizes(*shape)
    return _c_rmsnorm(x.data_ptr(), _mat("x", x, shape, dt, dev), _addr(residual), _mat("residual", residual, shape, dt, dev),
                      _vec("gamma", gamma, d, dt, dev), eps, _addr(x_out), _mat("x_out", x_out, shape, dt, dev),
                      _addr(y), _mat("y", y, shape, dt, dev), _addr(q), _mat("q", q, shape, torch.int8, dev),
                      _vec("q_scale", q_scale, T, torch.float32, dev), T, d, _CODES[dt], _launch_stream(stream, dev))


def packed_quantize_i8(x, q, scale, stream=None):
    """8-bit rows of x [T, d] (tokens, or a weight matrix): q int8 [T, d], scale float32 [T]."""
    st = _fast.packed_quantize_i8(x, q, scale, stream)
    if st is None:
        shape, dt, dev = x.shape, x.dtype, x.get_device()
        T, d = _sizes(*shape)
        st = _c_quantize_i8(x.data_ptr(), _mat("x", x, shape, dt, dev), _addr(q), _mat("q", q, shape, torch.int8, dev),
                            _vec("scale", scale, T, torch.float32, dev), T, d, _CODES[dt], _launch_stream(stream, dev))
    if st:
        _check("packed_quantize_i8", st)


def packed_linear_i8(x, x_scale, w, w_scale, y, bias=None, residual=None, act=RAG_ACT_NONE, stream=None):
    """y = act(x_scale w_scale (x w^T) + bias) + residual: x int8 [T, K] and w int8 [N, K] in 8-bit rows with
    their float32 scales ([T] and [N]); bias, residual and y (which may be residual) of one type."""
    st = _fast.packed_linear_i8(x, x_scale, w, w_scale, y, bias, residual, act, stream)
    if st is None:
        st = _checked_linear_i8(x, x_scale, w, w_scale, y, bias, residual, act, stream)
    if st:
        _check("packed_linear_i8", st)


def _checked_linear_i8(x, x_scale, w, w_scale, y, bias, residual, act, stream):
    dt, dev = y.dtype, y.get_device()
    T, K, N = _sizes(*x.shape, w.shape[0])
    if _mat("w", w, (N, K), torch.int8, dev) != K and N > 1:
        raise ValueError("w must be contiguous")
    return _c_linear_i8(x.data_ptr(), _mat("x", x, (T, K), torch.int8, dev), _vec("x_scale", x_scale, T, torch.float32, dev),
                        w.data_ptr(), _vec("w_scale", w_scale, N, torch.float32, dev), _vec("bias", bias, N, dt, dev),
                        _addr(residual), _mat("residual", residual, (T, N), dt, dev), _i32("act", act), y.data_ptr(),
                        _mat("y", y, (T, N), dt, dev), T, K, N, _CODES[dt], _launch_stream(stream, dev))


def rotary_frequencies(rot_dim, base=10000.0, scaling=RAG_ROTARY_PLAIN, factor=1.0, orig_len=0, beta_fast=32.0,
                       beta_slow=1.0):
    """(angle per position of each of rot_dim / 2 pairs, a float64 tensor on the CPU; amplitude)."""
    rot_dim, scaling, orig_len = _i32("rot_dim", rot_dim), _i32("scaling", scaling), _i32("orig_len", orig_len)
    f = torch.empty(min(max(rot_dim // 2, 1), RAG_ROTARY_MAX_DIM), dtype=torch.float64)  # (longer ones are refused)
    a = _f64()
    _check("rotary_frequencies", _c_rotary_frequencies(rot_dim, base, scaling, factor, orig_len, beta_fast, beta_slow,
                                                       _ptr(f), ctypes.addressof(a)))
    return f, a.value


def packed_rotary(plan: Plan, x, y, inv_freq, heads, head_dim=RAG_HEAD_DIM, layout=RAG_ROTARY_HALF, amplitude=1.0,
                  pos_start=None, inverse=False, stream=None):
    """Turns the first 2 * len(inv_freq) channels of each of `heads` heads of x [T, heads * head_dim] into y (which
    may be x).  inv_freq is a float64 device tensor; pos_start int32 [B] holds each sequence's first position;
    `inverse` turns back."""
    st = _fast.packed_rotary(plan, x, y, inv_freq, heads, head_dim, layout, amplitude, pos_start, inverse, stream)
    if st is None:
        dt, dev, n = x.dtype, x.get_device(), inv_freq.numel()
        shape = (plan.total_tokens, heads * head_dim)
        _sizes(2 * n)
        heads, head_dim, layout = _i32("heads", heads), _i32("head_dim", head_dim), _i32("layout", layout)
        st = _c_rotary(plan.ref(), x.data_ptr(), _mat("x", x, shape, dt, dev), y.data_ptr(), _mat("y", y, shape, dt, dev), heads,
                       head_dim, 2 * n, layout | (RAG_ROTARY_INVERSE if inverse else 0),
                       _vec("inv_freq", inv_freq, n, torch.float64, dev), amplitude,
                       _vec("pos_start", pos_start, plan.batch, torch.int32, dev), _CODES[dt], _launch_stream(stream, dev, plan))
    if st:
        _check("packed_rotary", st)


def ragged_attention_window_workspace(plan: Plan, max_kv_len, window, sinks=0, kv_heads=None, dtype=torch.bfloat16):
    """Workspace bytes of the two calls below (max_kv_len: plan.max_len for the first; may be 0)."""
    n = ctypes.c_size_t()
    _check("ragged_attention_window_workspace",
           _c_window_ws(plan.ref(), _bound("max_kv_len", max_kv_len), _i32("kv_heads", kv_heads or plan.heads),
                        _bound("window", window), _bound("sinks", sinks), _CODES[dtype], ctypes.byref(n)))
    return n.value


def _window_operands(plan, q, k, v, out, kv_rows, kv_heads, head_dim, workspace):
    """(dtype code, device, leading dimensions of q, k, v and out, workspace address and bytes)"""
    dt, dev = q.dtype, q.get_device()
    shape, kv = (plan.total_tokens, plan.heads * head_dim), (kv_rows, kv_heads * head_dim)
    lds = (_mat("q", q, shape, dt, dev), _mat("k", k, kv, dt, dev), _mat("v", v, kv, dt, dev), _mat("out", out, shape, dt, dev))
    if workspace is None:
        return _CODES[dt], dev, lds, None, 0
    if not workspace.is_contiguous() or workspace.get_device() != dev:
        raise ValueError("workspace must be contiguous and on the operands' device")
    return _CODES[dt], dev, lds, workspace.data_ptr(), workspace.numel() * workspace.element_size()


def ragged_attention_window(plan: Plan, q, k, v, out, scale, window, sinks=0, kv_heads=None, head_dim=RAG_HEAD_DIM,
                            workspace=None, stream=None):
    """Causal attention over the packed batch: position p sees keys j <= p with j > p - window or j < sinks.
    k and v hold kv_heads (default: all) heads, each shared by plan.heads / kv_heads query heads."""
    st = _fast.ragged_attention_window(plan, q, k, v, out, scale, window, sinks, kv_heads, head_dim, workspace, stream)
    if st is None:
        kvh, head_dim = _i32("kv_heads", kv_heads or plan.heads), _i32("head_dim", head_dim)
        code, dev, ld, ws, n = _window_operands(plan, q, k, v, out, plan.total_tokens, kvh, head_dim, workspace)
        st = _c_window(plan.ref(), q.data_ptr(), ld[0], k.data_ptr(), ld[1], v.data_ptr(), ld[2], kvh, head_dim, scale,
                       _bound("window", window), _bound("sinks", sinks), out.data_ptr(), ld[3], ws, n, code,
                       _launch_stream(stream, dev, plan))
    if st:
        _check("ragged_attention_window", st)


def ragged_attention_window_cached(plan: Plan, q, k, v, kv_first, kv_len, max_kv_len, out, scale, window, sinks=0,
                                   kv_heads=None, head_dim=RAG_HEAD_DIM, workspace=None, stream=None):
    """The same over caches k and v [rows, kv_heads * head_dim]: sequence b's keys are the kv_len[b] rows from
    kv_first[b] (int32 and int64 device tensors), its queries the last plan.lengths[b] of those positions."""
    st = _fast.ragged_attention_window_cached(plan, q, k, v, kv_first, kv_len, max_kv_len, out, scale, window, sinks, kv_heads,
                                              head_dim, workspace, stream)
    if st is None:
        kvh, head_dim, rows = _i32("kv_heads", kv_heads or plan.heads), _i32("head_dim", head_dim), k.shape[0]
        code, dev, ld, ws, n = _window_operands(plan, q, k, v, out, rows, kvh, head_dim, workspace)
        st = _c_window_cached(plan.ref(), q.data_ptr(), ld[0], k.data_ptr(), ld[1], v.data_ptr(), ld[2], rows,
                              _vec("kv_first", kv_first, plan.batch, torch.int64, dev),
                              _vec("kv_len", kv_len, plan.batch, torch.int32, dev), _bound("max_kv_len", max_kv_len), kvh,
                              head_dim, scale, _bound("window", window), _bound("sinks", sinks), out.data_ptr(), ld[3], ws, n, code,
                              _launch_stream(stream, dev, plan))
    if st:
        _check("ragged_attention_window_cached", st)


def encoder_layer_workspace(total_tokens, max_len, d_model, heads, d_ff, dtype=RAG_BF16, flags=0):
    n = ctypes.c_size_t()
    _check("encoder_layer_workspace", _c_ws(total_tokens, max_len, d_model, heads, d_ff, dtype, flags,
                                            ctypes.byref(n)))
    return n.value


WEIGHT_ORDER = ("w_qkv", "b_qkv", "w_o", "b_o", "ln1_g", "ln1_b", "w_ff1", "b_ff1", "w_ff2", "b_ff2", "ln2_g", "ln2_b")


def layer_weights(weights: dict) -> RagLayerWeights:
    return RagLayerWeights(*[weights[n].data_ptr() for n in WEIGHT_ORDER])


def encoder_layer(plan: Plan, x, y, weights, d_ff, workspace, heads=None, head_dim=RAG_HEAD_DIM, ln_eps=1e-5,
                  act=RAG_ACT_GELU_ERF, flags=0, stream=None, events=None):
    """`weights`: dict of device tensors (WEIGHT_ORDER names) or a RagLayerWeights;
    `events`: optional ctypes array of RAG_LAYER_EVENTS hipEvent_t handles."""
    T, d = x.shape
    heads = plan.heads if heads is None else heads
    w = weights if isinstance(weights, RagLayerWeights) else layer_weights(weights)
    _check("encoder_layer", _c_layer(plan.ref(), _ptr(x), _ptr(y), d, heads, head_dim, d_ff, ln_eps, act, flags,
                                     ctypes.byref(w), _ptr(workspace), workspace.numel() * workspace.element_size(),
                                     _dtype_code(x), _stream(stream),
                                     None if events is None else ctypes.cast(events, ctypes.c_void_p)))


def encoder_layer_noalloc(plan: Plan, x, y, weights, d_ff, heads=None, head_dim=RAG_HEAD_DIM, ln_eps=1e-5,
                          act=RAG_ACT_GELU_ERF, flags=0, stream=None):
    """encoder_layer with the library's fixed device scratch array as its workspace
    (RAG_NOALLOC_SCRATCH_BYTES): no workspace argument, nothing allocated."""
    T, d = x.shape
    heads = plan.heads if heads is None else heads
    w = weights if isinstance(weights, RagLayerWeights) else layer_weights(weights)
    _check("encoder_layer_noalloc", _c_layer_noalloc(plan.ref(), _ptr(x), _ptr(y), d, heads, head_dim, d_ff, ln_eps,
                                                     act, flags, ctypes.byref(w), _dtype_code(x), _stream(stream)))


def vgemm_plan_capacity(batch, max_m, max_n):
    n = _i64()
    _check("vgemm_plan_capacity", _c_vgemm_capacity(batch, max_m, max_n, ctypes.byref(n)))
    return n.value


def vgemm_tile_count(host_dims):
    """Exact tile count of a batch from its (m, n, k) sizes held on the host."""
    import numpy as np

    d = np.ascontiguousarray(np.asarray(host_dims, dtype=np.int32).reshape(-1, 3))
    n = _i64()
    _check("vgemm_tile_count", _c_vgemm_tile_count(d.shape[0], d.ctypes.data_as(ctypes.c_void_p), ctypes.byref(n)))
    return n.value


class VgemmPlan:
    """Device arrays of a vgemm batch's prelude, allocated with torch.

    `dims` is an int32 device tensor [B, 3] of (m, n, k).  `tile_cap` defaults to
    the exact tile count when `host_dims` (the same sizes on the host) is given,
    else to the bound from `max_m` / `max_n`."""

    def __init__(self, dims: torch.Tensor, tile_cap: int | None = None, host_dims=None, max_m=None, max_n=None):
        if dims.dtype != torch.int32 or not dims.is_cuda or dims.dim() != 2 or dims.shape[1] != 3:
            raise ValueError("dims must be a [B, 3] int32 device tensor")
        if not dims.is_contiguous():
            raise ValueError("dims must be contiguous")
        dev = dims.device
        B = dims.shape[0]
        if tile_cap is None:
            if host_dims is not None:
                tile_cap = vgemm_tile_count(host_dims)
            elif max_m is not None and max_n is not None:
                tile_cap = vgemm_plan_capacity(B, max_m, max_n)
            else:
                raise ValueError("give tile_cap, host_dims or max_m and max_n")
        i64 = dict(dtype=torch.int64, device=dev)
        self.dims = dims
        self.a_off, self.b_off, self.c_off = (torch.empty(B + 1, **i64) for _ in range(3))
        self.order = torch.empty(B, dtype=torch.int32, device=dev)
        self.tile_off = torch.empty(B + 1, **i64)
        self.tile_items = torch.empty(max(4 * tile_cap, 4), dtype=torch.int32, device=dev)
        self.status = torch.zeros(3, dtype=torch.int32, device=dev)
        self.batch, self.tile_cap = B, tile_cap
        self.c = RagVgemmPlan(B, tile_cap, dims.data_ptr(), self.a_off.data_ptr(), self.b_off.data_ptr(),
                              self.c_off.data_ptr(), self.order.data_ptr(), self.tile_off.data_ptr(),
                              self.tile_items.data_ptr(), self.status.data_ptr())

    def ref(self):
        return ctypes.byref(self.c)

    def data_errors(self):
        """Decode status[0] (synchronises)."""
        f = int(self.status[0].item())
        return [msg for bit, msg in VGEMM_DATA_BITS.items() if f & bit]

    def n_tiles(self):
        return int(self.status[1].item())


def vgemm_offsets(plan: VgemmPlan, stream=None):
    _check("vgemm_offsets", _c_vgemm_offsets(plan.ref(), _stream(stream)))


def ragged_vgemm(plan: VgemmPlan, a, b, c, stream=None):
    """C_b = A_b B_b^T for every problem of the packed batch: a, b, c are 1-D
    tensors of one dtype holding the packed operands."""
    if not (a.dtype == b.dtype == c.dtype):
        raise TypeError("a, b and c must share one dtype")
    for t in (a, b, c):
        if not t.is_contiguous():
            raise ValueError("a, b and c must be contiguous")
    _check("ragged_vgemm", _c_vgemm(plan.ref(), _ptr(a), a.numel(), _ptr(b), b.numel(), _ptr(c), c.numel(),
                                    _dtype_code(a), _stream(stream)))


def ragged_trmm(l, b, c, stream=None):
    """C = tril(L) B: l [n, n], b and c [n, m], 2-D tensors of one dtype with unit
    column stride (entries of l above the diagonal are ignored)."""
    n, m = b.shape
    if l.shape[0] != n or l.shape[1] < n or c.shape != b.shape:
        raise ValueError("expected l [n, n], b [n, m] and c [n, m]")
    if not (l.dtype == b.dtype == c.dtype):
        raise TypeError("l, b and c must share one dtype")
    _check("ragged_trmm", _c_trmm(_ptr(l), _ld(l), _ptr(b), _ld(b), _ptr(c), _ld(c), n, m, _dtype_code(b),
                                  _stream(stream)))
