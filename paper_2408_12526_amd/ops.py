"""Thin binding over the operators of libsp_mi355x.so that stand by themselves (include/sp_ops.h): products in 8-bit
integers, rotary positions, and attention with capped scores, distance biases and masks.

Argument marshalling and checks only: torch supplies device memory and streams, every step runs in the library's kernels, and there
is no fallback.  A call runs on the current stream of the tensors' device, allocates its outputs and workspace from torch's
allocator, waits for nothing and can be captured in a graph.  What torch must know for the kernels to stay inside the tensors (shapes,
types, devices, strides) is checked here and raises ValueError; what the library refuses raises sp.SpError.  None has a
gradient: inputs that require one are refused while gradients are recorded.
"""
from __future__ import annotations

import ctypes as C
import math

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
    lib.sp_attention_workspace_bytes.restype = sz; lib.sp_attention_workspace_bytes.argtypes = [C.POINTER(sp_attention_args)]
    lib.sp_attention.restype = C.c_int; lib.sp_attention.argtypes = [C.POINTER(sp_attention_args), vp, sz, vp]
    return lib


_lib = _load()
_check = _sp._check


def _need(ok: bool, what: str) -> None:
    if not ok:
        raise ValueError(what)


def _home(first: torch.Tensor, *others) -> torch.device:
    """The device that all tensors are on."""
    dev = first.device
    _need(dev.type == "cuda", "the tensors have to be on a GPU: there is no CPU path in this library")
    recording = torch.is_grad_enabled()
    for t in (first, *others):
        if t is not None:
            _need(t.device == dev, f"tensors on {t.device} and {dev}")
            _need(not (recording and t.requires_grad), "this operator has no gradient: call it under torch.no_grad() or on detached tensors")
    return dev


class _On:
    """The device made current for the call where it is not (a context manager; nothing is done in the usual case)."""
    __slots__ = ("index", "before")

    def __init__(self, dev: torch.device):
        self.index = dev.index

    def __enter__(self):
        self.before = torch.cuda.current_device()
        if self.before != self.index:
            torch.cuda.set_device(self.index)
        return torch.cuda.current_stream(self.index).cuda_stream

    def __exit__(self, *_):
        if self.before != self.index:
            torch.cuda.set_device(self.before)


def _dtype(t: torch.Tensor) -> int:
    d = _DTYPES.get(t.dtype)
    _need(d is not None, f"float32 or bfloat16 is wanted, not {t.dtype}")
    return d


def _vector(t, name: str, dtype, n: int):
    if t is None:
        return None
    _need(t.dtype == dtype and t.dim() == 1 and t.numel() == n and t.is_contiguous(), f"{name}: a contiguous {dtype} vector of {n} is wanted")
    return t.data_ptr()


def _rows(t: torch.Tensor, name: str, shape, dtype) -> int:
    """The row stride of a matrix whose rows are contiguous."""
    _need(t.dtype == dtype and tuple(t.shape) == tuple(shape), f"{name}: {dtype} of shape {tuple(shape)} is wanted, not {t.dtype} {tuple(t.shape)}")
    _need(t.shape[1] <= 1 or t.stride(1) == 1, f"{name}: the elements of a row have to be contiguous")
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


# ---- 8-bit integers ---------------------------------------------------------------------------------------------

def quantize_int8(x: torch.Tensor):
    """Rows of x [rows, width] as (codes int8 [rows, width], scales float32 [rows]), x ~ codes * scales: scale = max |row| / 127.
    The codes' rows lie at multiples of 16 bytes with zeros behind them, as linear_int8 wants its weights."""
    dtype, dev = _dtype(x), _home(x)
    _need(x.dim() == 2 and x.shape[1] >= 1, "x: a matrix is wanted")
    rows, width = x.shape
    x_row = _rows(x, "x", x.shape, x.dtype)
    pad = (width + 15) // 16 * 16
    with _On(dev) as stream:
        codes = torch.empty(rows, pad, dtype=torch.int8, device=dev)
        if pad > width:
            codes[:, width:].zero_()
        scales = torch.empty(rows, dtype=torch.float32, device=dev)
        _check(_lib.sp_quantize_int8(x.data_ptr(), x_row, dtype, rows, width, codes.data_ptr(), pad, scales.data_ptr(), stream))
    return codes[:, :width], scales


def linear_int8(x: torch.Tensor, codes: torch.Tensor, scales: torch.Tensor, bias: torch.Tensor | None = None, *,
                residual: torch.Tensor | None = None, gelu: bool = False, out: torch.Tensor | None = None) -> torch.Tensor:
    """x [tokens, width_in] (float32 or bfloat16) times the weights codes [width_out, width_in] (int8) * scales [width_out], the rows of
    x quantised to 8-bit integers with a scale each on the way; + bias (float32), then GELU, or + residual.  Returns out
    [tokens, width_out] of x's type.  The rows of codes start at multiples of 16 bytes (quantize_int8 lays them out so)."""
    dtype, dev = _dtype(x), _home(x, codes, scales, bias, residual, out)
    _need(x.dim() == 2 and codes.dim() == 2, "x and codes: matrices are wanted")
    T, K = x.shape
    N = codes.shape[0]
    _need(codes.dtype == torch.int8 and codes.shape[1] == K, f"codes: int8 [width_out, {K}] is wanted")
    _need(K >= 1 and N >= 1, "codes: at least one row and one column are wanted")
    pad = (K + 15) // 16 * 16
    w_row = codes.stride(0) if N > 1 else pad
    _need(K == 1 or codes.stride(1) == 1, "codes: the elements of a row have to be contiguous")
    _need(w_row % 16 == 0 and codes.data_ptr() % 16 == 0, "codes: rows have to start at multiples of 16 bytes (see quantize_int8)")
    _need((N - 1) * w_row + pad + codes.storage_offset() <= codes.untyped_storage().nbytes(),
          "codes: the last row's storage has to reach to the next multiple of 16 (see quantize_int8)")
    _need(not (gelu and residual is not None), "gelu or residual, not both")
    x_row = _rows(x, "x", (T, K), x.dtype)
    r_row = _rows(residual, "residual", (T, N), x.dtype) if residual is not None else 0
    sc, bi = _vector(scales, "scales", torch.float32, N), _vector(bias, "bias", torch.float32, N)
    with _On(dev) as stream:
        if out is None:
            out = torch.empty(T, N, dtype=x.dtype, device=dev)
        o_row = _rows(out, "out", (T, N), x.dtype)
        need = _lib.sp_linear_int8_workspace_bytes(T, K)
        ws = torch.empty(need, dtype=torch.uint8, device=dev)
        _check(_lib.sp_linear_int8(x.data_ptr(), x_row, dtype, T, K, codes.data_ptr(), w_row, sc, N, bi,
                                   LINEAR_GELU if gelu else LINEAR_RESIDUAL if residual is not None else LINEAR_PLAIN,
                                   residual.data_ptr() if residual is not None else None, r_row, out.data_ptr(), o_row, ws.data_ptr(), need, stream))
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
    _need(layout in ROTARY_LAYOUTS, f"layout: one of {', '.join(ROTARY_LAYOUTS)}")
    _need((positions is None) != (cu_seqlens is None), "positions or cu_seqlens: one of the two")
    T, A, D = x.shape
    _need(x.stride(2) == 1, "x: the elements of a head have to be contiguous")
    fr = _vector(frequencies, "frequencies", torch.float64, frequencies.numel())
    pos = _vector(positions, "positions", torch.int32, T)
    batch, cu = 0, None
    if cu_seqlens is not None:
        batch = cu_seqlens.numel() - 1
        _need(batch >= 0, "cu_seqlens: [batch + 1] is wanted")
        cu = _vector(cu_seqlens, "cu_seqlens", torch.int32, batch + 1)
    with _On(dev) as stream:
        if out is None:
            out = torch.empty(T, A, D, dtype=x.dtype, device=dev)
        _need(out.dtype == x.dtype and out.shape == x.shape and out.stride(2) == 1, "out: like x")
        _check(_lib.sp_rotary(x.data_ptr(), x.stride(0), x.stride(1), out.data_ptr(), out.stride(0), out.stride(1), dtype, T, A, D,
                              2 * frequencies.numel(), ROTARY_LAYOUTS[layout], fr, float(factor), pos, cu, batch, stream))
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
    Tk, G = k.shape[0], k.shape[1]
    _need(k.dtype == q.dtype and v.dtype == q.dtype and k.shape[2] == D and v.shape == k.shape, "k and v: of q's type and width, and of one shape")
    _need(q.stride(2) == 1 and k.stride(2) == 1 and v.stride(2) == 1, "q, k, v: the elements of a head have to be contiguous")
    batch = cu_q.numel() - 1
    _need(batch >= 0, "cu_q: [batch + 1] is wanted")
    if cu_k is None:
        _need(Tk == Tq, "cu_k is wanted where queries and keys differ in number")
        cu_k, max_k = cu_q, max_q if max_k is None else max_k
        doc_k = doc_q if doc_k is None else doc_k
    _need(max_k is not None, "max_k is wanted with cu_k")
    _need((doc_q is None) == (doc_k is None), "doc_q and doc_k: both or none")
    left, right = (-1, -1) if window is None else (int(window[0]), int(window[1]))
    if causal:
        _need(right <= 0, "causal: no keys to the right")
        right = 0
    reach = 0
    if bias is not None:
        _need(bias.dtype == torch.float32 and bias.dim() == 2 and bias.shape[0] == A and bias.shape[1] % 2 == 1 and bias.is_contiguous(),
              f"bias: contiguous float32 [{A}, 2 reach + 1] is wanted")
        reach = bias.shape[1] // 2
    a = sp_attention_args(
        q=q.data_ptr(), k=k.data_ptr(), v=v.data_ptr(), q_token=q.stride(0), q_head=q.stride(1), k_token=k.stride(0), k_head=k.stride(1),
        v_token=v.stride(0), v_head=v.stride(1), cu_q=_vector(cu_q, "cu_q", torch.int32, batch + 1), cu_k=_vector(cu_k, "cu_k", torch.int32, batch + 1),
        dtype=dtype, batch=batch, heads=A, kv_heads=G, width=D, total_q=Tq, total_k=Tk, max_q=int(max_q), max_k=int(max_k),
        scale=1.0 / math.sqrt(D) if scale is None else float(scale), cap=float(cap), left=max(left, -1), right=max(right, -1),
        prefix=_vector(prefix, "prefix", torch.int32, batch), q_first=_vector(q_first, "q_first", torch.int32, batch),
        doc_q=_vector(doc_q, "doc_q", torch.int32, Tq), doc_k=_vector(doc_k, "doc_k", torch.int32, Tk),
        slopes=_vector(slopes, "slopes", torch.float32, A), bias=bias.data_ptr() if bias is not None else None, reach=reach)
    with _On(dev) as stream:
        lse = None
        if out is None:
            out = torch.empty(Tq, A, D, dtype=q.dtype, device=dev)
        else:
            _need(out.dtype == q.dtype and out.shape == q.shape and out.stride(2) == 1, "out: like q")
        a.out, a.out_token, a.out_head = out.data_ptr(), out.stride(0), out.stride(1)
        if with_lse:
            lse = torch.empty(Tq, A, dtype=torch.float32, device=dev)
            a.lse = lse.data_ptr()
        need = _lib.sp_attention_workspace_bytes(C.byref(a))
        ws = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
        _check(_lib.sp_attention(C.byref(a), ws.data_ptr() if need else None, need, stream))
    return (out, lse) if with_lse else out
