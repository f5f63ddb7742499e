"""Thin binding over the operators of libsp_mi355x.so that stand by themselves (include/sp_ops.h): products in 8-bit
integers, rotary positions, and attention with capped scores, distance biases and masks.

Argument marshalling and checks only: torch supplies device memory and streams, every step runs in the library's kernels, and there
is no fallback.  A call runs on the current stream of the tensors' device, allocates its outputs and workspace from torch's
allocator, waits for nothing and can be captured in a graph.  What torch must know for the kernels to stay inside the tensors (shapes,
types, devices, strides) is checked here and raises ValueError; what the library refuses raises sp.SpError.  None has a
gradient: inputs that require one are refused while gradients are recorded, inputs with a tangent (forward mode) always.
"""
from __future__ import annotations

import ctypes as C
import functools
import math
import struct

import numpy as np
import torch

from . import sp as _sp
from .sp import SpError  # noqa: F401

LINEAR_PLAIN, LINEAR_GELU, LINEAR_RESIDUAL = 0, 1, 2
ROTARY_LAYOUTS = {"half": 0, "interleaved": 1}
ROTARY_SCALINGS = {"none": 0, "linear": 1, "ntk": 2, "parts": 3}
_DTYPES = {torch.float32: _sp.SP_DTYPE_FP32, torch.bfloat16: _sp.SP_DTYPE_BF16}


class sp_attention_args(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("q", "k", "v", "out", "lse")] + [
        (n, C.c_int64) for n in ("q_token", "q_head", "k_token", "k_head", "v_token", "v_head", "out_token", "out_head")] + [
        (n, C.c_void_p) for n in ("cu_q", "cu_k")] + [
        (n, C.c_int32) for n in ("dtype", "batch", "heads", "kv_heads", "width", "total_q", "total_k", "max_q", "max_k")] + [
        ("scale", C.c_float), ("cap", C.c_float), ("left", C.c_int32), ("right", C.c_int32)] + [
        (n, C.c_void_p) for n in ("prefix", "q_first", "doc_q", "doc_k", "slopes", "bias")] + [("reach", C.c_int32)]


# The same for struct.pack, which fills it several times faster than the fields one by one.
_ATTENTION = struct.Struct("@5P8q2P9i2f2i6Pi0P")
assert _ATTENTION.size == C.sizeof(sp_attention_args)


def _load() -> C.CDLL:
    lib = _sp.raw_lib()
    vp, i32, i64, sz, f32, f64 = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t, C.c_float, C.c_double
    lib.sp_quantize_int8.restype = C.c_int; lib.sp_quantize_int8.argtypes = [vp, i64, i32, i32, i32, vp, i64, vp, vp]
    lib.sp_linear_int8_workspace_bytes.restype = sz; lib.sp_linear_int8_workspace_bytes.argtypes = [i32, i32]
    lib.sp_linear_int8.restype = C.c_int
    lib.sp_linear_int8.argtypes = [vp, i64, i32, i32, i32, vp, i64, vp, i32, vp, i32, vp, i64, vp, i64, vp, sz, vp]
    lib.sp_rotary_frequencies.restype = C.c_int
    lib.sp_rotary_frequencies.argtypes = [i32, f64, i32, f64, f64, vp, C.POINTER(f32)]
    lib.sp_rotary.restype = C.c_int
    lib.sp_rotary.argtypes = [vp, i64, i64, vp, i64, i64, i32, i32, i32, i32, i32, i32, vp, f32, vp, vp, i32, vp]
    lib.sp_attention_workspace_bytes.restype = sz; lib.sp_attention_workspace_bytes.argtypes = [vp]
    lib.sp_attention.restype = C.c_int; lib.sp_attention.argtypes = [vp, vp, sz, vp]
    return lib


_lib = _load()
_check = _sp._check


def _need(ok: bool, what: str) -> None:
    if not ok:
        raise ValueError(what)


_raw_stream = torch._C._cuda_getCurrentRawStream
_recording = torch.is_grad_enabled
_forward_ad = torch.autograd.forward_ad
_bytes_of = functools.lru_cache(maxsize=4096)(_lib.sp_linear_int8_workspace_bytes)


def _home(first: torch.Tensor, *others) -> int:
    """The index of the device that all tensors are on."""
    dev = first.get_device()
    _need(dev >= 0, "the tensors have to be on a GPU: there is no CPU path in this library")
    if _forward_ad._current_level >= 0:
        for t in (first, *others):
            if t is not None and t.is_floating_point() and _forward_ad.unpack_dual(t).tangent is not None:
                raise ValueError("this operator has no gradient: call it on detached tensors")
    recording = _recording()
    if recording and first.requires_grad:
        raise ValueError("this operator has no gradient: call it under torch.no_grad() or on detached tensors")
    for t in others:
        if t is not None:
            if t.get_device() != dev:
                raise ValueError(f"tensors on {t.device} and {first.device}")
            if recording and t.requires_grad:
                raise ValueError("this operator has no gradient: call it under torch.no_grad() or on detached tensors")
    return dev


class _On:
    """The device made current for the call where it is not."""
    __slots__ = ("index", "before")

    def __init__(self, index: int):
        self.index = index

    def __enter__(self):
        self.before = torch.cuda.current_device()
        torch.cuda.set_device(self.index)

    def __exit__(self, *_):
        torch.cuda.set_device(self.before)


def _call(dev: int, fn, *args) -> None:
    """fn(*args, stream) on the current stream of the device, with the device current."""
    if torch._C._cuda_getDevice() == dev:
        rc = fn(*args, _raw_stream(dev))
    else:
        with _On(dev):
            rc = fn(*args, _raw_stream(dev))
    if rc:
        raise SpError(rc)


def _fit(*sizes: int) -> None:
    """Sizes that the library takes as 32-bit numbers."""
    if max(sizes) > 0x7fffffff:
        raise ValueError(f"sizes of 2^31 and more are not taken: {sizes}")


def _dtype(t: torch.Tensor) -> int:
    d = _DTYPES.get(t.dtype)
    if d is None:
        raise ValueError(f"float32 or bfloat16 is wanted, not {t.dtype}")
    return d


def _vector(t, name: str, dtype, n: int):
    if t is None:
        return None
    if t.dtype is not dtype or t.dim() != 1 or t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{name}: a contiguous {dtype} vector of {n} is wanted")
    return t.data_ptr()


def _rows(t: torch.Tensor, name: str, shape, dtype) -> int:
    """The row stride of a matrix whose rows are contiguous."""
    if t.dtype is not dtype or t.shape != shape:
        raise ValueError(f"{name}: {dtype} of shape {tuple(shape)} is wanted, not {t.dtype} {tuple(t.shape)}")
    row, one = t.stride()
    if one != 1 and shape[1] > 1:
        raise ValueError(f"{name}: the elements of a row have to be contiguous")
    return row if shape[0] > 1 else shape[1]


# ---- 8-bit integers ---------------------------------------------------------------------------------------------

def quantize_int8(x: torch.Tensor):
    """Rows of x [rows, width] as (codes int8 [rows, width], scales float32 [rows]), x ~ codes * scales: scale = max |row| / 127.
    The codes' rows lie at multiples of 16 bytes with zeros behind them, as linear_int8 wants its weights."""
    dtype, dev = _dtype(x), _home(x)
    _need(x.dim() == 2 and x.shape[1] >= 1, "x: a matrix is wanted")
    rows, width = x.shape
    _fit(rows, width)
    x_row = _rows(x, "x", x.shape, x.dtype)
    pad = (width + 15) // 16 * 16
    codes = torch.empty(rows, pad, dtype=torch.int8, device=x.device)
    if pad > width:
        codes[:, width:].zero_()
    scales = torch.empty(rows, dtype=torch.float32, device=x.device)
    _call(dev, _lib.sp_quantize_int8, x.data_ptr(), x_row, dtype, rows, width, codes.data_ptr(), pad, scales.data_ptr())
    return codes[:, :width], scales


def linear_int8(x: torch.Tensor, codes: torch.Tensor, scales: torch.Tensor, bias: torch.Tensor | None = None, *,
                residual: torch.Tensor | None = None, gelu: bool = False, out: torch.Tensor | None = None) -> torch.Tensor:
    """x [tokens, width_in] (float32 or bfloat16) times the weights codes [width_out, width_in] (int8) * scales [width_out], the rows of
    x quantised to 8-bit integers with a scale each on the way; + bias (float32), then GELU, or + residual.  Returns out
    [tokens, width_out] of x's type.  The rows of codes start at multiples of 16 bytes (quantize_int8 lays them out so)."""
    dtype, dev = _dtype(x), _home(x, codes, scales, bias, residual, out)
    _need(x.dim() == 2 and codes.dim() == 2, "x and codes: matrices are wanted")
    T, K = x.shape
    N, Kw = codes.shape
    _fit(T, K, N)
    _need(codes.dtype is torch.int8 and Kw == K, "codes: int8 [width_out, width_in] is wanted")
    _need(K >= 1 and N >= 1, "codes: at least one row and one column are wanted")
    pad = (K + 15) // 16 * 16
    w_row, w_one = codes.stride()
    if N == 1:
        w_row = pad
    w = codes.data_ptr()
    _need(K == 1 or w_one == 1, "codes: the elements of a row have to be contiguous")
    _need(w_row % 16 == 0 and w % 16 == 0, "codes: rows have to start at multiples of 16 bytes (see quantize_int8)")
    _need(pad == K or (N - 1) * w_row + pad + codes.storage_offset() <= codes.untyped_storage().nbytes(),
          "codes: the last row's storage has to reach to the next multiple of 16 (see quantize_int8)")
    _need(not (gelu and residual is not None), "gelu or residual, not both")
    shape = (T, N)
    x_row = _rows(x, "x", x.shape, x.dtype)
    r, r_row, epilogue = None, 0, LINEAR_GELU if gelu else LINEAR_PLAIN
    if residual is not None:
        r, r_row, epilogue = residual.data_ptr(), _rows(residual, "residual", shape, x.dtype), LINEAR_RESIDUAL
    sc, bi = _vector(scales, "scales", torch.float32, N), _vector(bias, "bias", torch.float32, N)
    if out is None:
        out, o_row = x.new_empty(shape), N
    else:
        o_row = _rows(out, "out", shape, x.dtype)
    need = _bytes_of(T, K)
    ws = torch.empty(need, dtype=torch.uint8, device=x.device)
    _call(dev, _lib.sp_linear_int8, x.data_ptr(), x_row, dtype, T, K, w, w_row, sc, N, bi, epilogue, r, r_row, out.data_ptr(), o_row,
          ws.data_ptr(), need)
    return out


# ---- rotary positions -------------------------------------------------------------------------------------------

def rotary_frequencies(dim: int, base: float = 10000.0, scaling: str = "none", factor: float = 1.0, trained: float = 4096.0):
    """(frequencies float64 [dim / 2], the factor on the rotated values) for rotary(): numpy and a number, on the host.  scaling, for
    contexts `factor` times as long as the `trained` one: "none", "linear", "ntk" or "parts" (see include/sp_ops.h)."""
    _need(scaling in ROTARY_SCALINGS, f"scaling: one of {', '.join(ROTARY_SCALINGS)}")
    f = np.empty(max(1, int(dim) // 2), np.float64)
    on_values = C.c_float()
    _check(_lib.sp_rotary_frequencies(int(dim), float(base), ROTARY_SCALINGS[scaling], float(factor), float(trained), f.ctypes.data, C.byref(on_values)))
    return f, float(on_values.value)


def rotary(x: torch.Tensor, frequencies: torch.Tensor, *, positions: torch.Tensor | None = None, cu_seqlens: torch.Tensor | None = None,
           layout: str = "half", factor: float = 1.0, out: torch.Tensor | None = None) -> torch.Tensor:
    """x [tokens, heads, width] with the first 2 * len(frequencies) elements of every head rotated by position * frequency, times factor.
    positions int32 [tokens], or cu_seqlens int32 [batch + 1] (a token's position is its index in its sequence).  out may be x: then
    in place.  Tokens of no sequence stay as they were in `out` and are unspecified in an output that is made here."""
    dtype, dev = _dtype(x), _home(x, frequencies, positions, cu_seqlens, out)
    _need(x.dim() == 3 and x.shape[1] >= 1 and x.shape[2] >= 2, "x: [tokens, heads, width] is wanted")
    way = ROTARY_LAYOUTS.get(layout)
    _need(way is not None, "layout: half or interleaved")
    _need((positions is None) != (cu_seqlens is None), "positions or cu_seqlens: one of the two")
    T, A, D = x.shape
    _fit(T, A, D)
    x_token, x_head, one = x.stride()
    _need(one == 1, "x: the elements of a head have to be contiguous")
    half = frequencies.numel()
    fr = _vector(frequencies, "frequencies", torch.float64, half)
    batch, pos, cu = 0, None, None
    if positions is not None:
        pos = _vector(positions, "positions", torch.int32, T)
    else:
        batch = cu_seqlens.numel() - 1
        _need(batch >= 0, "cu_seqlens: [batch + 1] is wanted")
        cu = _vector(cu_seqlens, "cu_seqlens", torch.int32, batch + 1)
    if out is None:
        out, o_token, o_head = x.new_empty((T, A, D)), A * D, D
    else:
        _need(out.dtype is x.dtype and out.shape == x.shape and out.stride(2) == 1, "out: like x")
        o_token, o_head, _ = out.stride()
    _call(dev, _lib.sp_rotary, x.data_ptr(), x_token, x_head, out.data_ptr(), o_token, o_head, dtype, T, A, D, 2 * half, way, fr, factor, pos, cu, batch)
    return out


# ---- attention --------------------------------------------------------------------------------------------------

def attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, cu_q: torch.Tensor, max_q: int, cu_k: torch.Tensor | None = None,
              max_k: int | None = None, *, scale: float | None = None, cap: float = 0.0, causal: bool = False, window=None,
              prefix: torch.Tensor | None = None, q_first: torch.Tensor | None = None, doc_q: torch.Tensor | None = None,
              doc_k: torch.Tensor | None = None, slopes: torch.Tensor | None = None, bias: torch.Tensor | None = None,
              out: torch.Tensor | None = None, with_lse: bool = False):
    """softmax(scores) v over packed sequences; the definition is in include/sp_ops.h.
    q [total_q, heads, width], k and v [total_k, kv_heads, width] (float32 or bfloat16, heads contiguous, strides of 16-byte multiples);
    cu_q, cu_k int32 [batch + 1] (cu_k: cu_q), max_q, max_k upper bounds on the lengths (max_k: max_q).
    scale (1 / sqrt(width)) and cap (0: none) of the scores; causal, window (left, right) and prefix int32 [batch] say which distances are
    seen, -1 being no bound; q_first int32 [batch] is the position of a sequence's first query (its queries are the last); doc_q, doc_k int32
    [total] documents (doc_k: doc_q); slopes float32 [heads], bias float32 [heads, 2 reach + 1] by distance.
    Returns out [total_q, heads, width], and with with_lse the logarithm of the sums, float32 [total_q, heads].  Rows of no sequence
    stay as they were in `out` and are unspecified in outputs that are made here."""
    dev = _home(q, k, v, cu_q, cu_k, prefix, q_first, doc_q, doc_k, slopes, bias, out)
    dtype = _dtype(q)
    _need(q.dim() == 3 and k.dim() == 3 and v.dim() == 3, "q, k, v: [tokens, heads, width] is wanted")
    Tq, A, D = q.shape
    Tk, G, Dk = k.shape
    _need(k.dtype is q.dtype and v.dtype is q.dtype and Dk == D and v.shape == k.shape, "k and v: of q's type and width, and of one shape")
    (q_token, q_head, q1), (k_token, k_head, k1), (v_token, v_head, v1) = q.stride(), k.stride(), v.stride()
    _need(q1 == k1 == v1 == 1, "q, k, v: the elements of a head have to be contiguous")
    batch = cu_q.numel() - 1
    _need(batch >= 0, "cu_q: [batch + 1] is wanted")
    if cu_k is None:
        _need(Tk == Tq, "cu_k is wanted where queries and keys differ in number")
        cu_k, max_k = cu_q, max_q if max_k is None else max_k
        doc_k = doc_q if doc_k is None else doc_k
    _need(max_k is not None, "max_k is wanted with cu_k")
    _need((doc_q is None) == (doc_k is None), "doc_q and doc_k: both or none")
    left, right = (-1, -1) if window is None else window
    if causal:
        _need(right <= 0, "causal: no keys to the right")
        right = 0
    reach, bi = 0, None
    if bias is not None:
        _need(bias.dtype is torch.float32 and bias.dim() == 2 and bias.shape[0] == A and bias.shape[1] % 2 == 1 and bias.is_contiguous(),
              "bias: contiguous float32 [heads, 2 reach + 1] is wanted")
        reach, bi = bias.shape[1] // 2, bias.data_ptr()
    if out is None:
        out, o_token, o_head = q.new_empty((Tq, A, D)), A * D, D
    else:
        _need(out.dtype is q.dtype and out.shape == q.shape and out.stride(2) == 1, "out: like q")
        o_token, o_head, _ = out.stride()
    lse = torch.empty((Tq, A), dtype=torch.float32, device=q.device) if with_lse else None
    try:
        args = _ATTENTION.pack(
            q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), lse.data_ptr() if with_lse else 0, q_token, q_head, k_token, k_head, v_token, v_head,
            o_token, o_head, _vector(cu_q, "cu_q", torch.int32, batch + 1), _vector(cu_k, "cu_k", torch.int32, batch + 1), dtype, batch, A, G, D, Tq, Tk,
            max_q, max_k, 1.0 / math.sqrt(D) if scale is None else scale, cap, left if left > -1 else -1, right if right > -1 else -1,
            _vector(prefix, "prefix", torch.int32, batch) or 0, _vector(q_first, "q_first", torch.int32, batch) or 0,
            _vector(doc_q, "doc_q", torch.int32, Tq) or 0, _vector(doc_k, "doc_k", torch.int32, Tk) or 0,
            _vector(slopes, "slopes", torch.float32, A) or 0, bi or 0, reach)
    except (struct.error, OverflowError, TypeError) as e:
        raise ValueError(f"a size or number that does not fit its field: {e}") from None
    need = _lib.sp_attention_workspace_bytes(args)
    ws = torch.empty(need, dtype=torch.uint8, device=q.device) if need else None      # (held until the launches are enqueued)
    _call(dev, _lib.sp_attention, args, None if ws is None else ws.data_ptr(), need)
    return (out, lse) if with_lse else out
