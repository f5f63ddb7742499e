"""The operators of include/sp_ops.h in numpy and 64 bits, one row after another, with bounds on what fp32 arithmetic may be off.

Independent of the library.  Inputs are numpy arrays of the values the library is given (bfloat16 ones as float32).
"""
from __future__ import annotations

import math

import numpy as np
import torch

HALF_STEP = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}     # of a rounding, relative to the value
F32 = 2.0 ** -24


def quantize(x):
    """codes (float64), scales (float64) of the rows: single fp32 operations."""
    x = np.asarray(x, np.float32)
    codes, scales = np.zeros(x.shape, np.float64), np.zeros(len(x), np.float64)
    for t, row in enumerate(x):
        a = np.abs(row).max()
        if not np.isfinite(row).all():
            scales[t] = math.nan
        elif a >= np.float32(2.0 ** -100):
            scales[t] = a / np.float32(127)
            codes[t] = np.rint(row * (np.float32(127) / a))
    return codes, scales


def linear_int8(x, w_codes, w_scales, bias=None, residual=None, gelu=False, dtype="fp32"):
    """(y, bound): every fp32 operation behind the integer sum off by at most half a step of its result, doubled for the
    order; GELU to 4e-7 (its slope is at most 1.13); the rounding to dtype."""
    codes, scales = quantize(x)
    y = (codes @ np.asarray(w_codes, np.float64).T) * scales[:, None] * np.asarray(w_scales, np.float64)
    off = 8 * F32 * np.abs(y)
    if bias is not None:
        y = y + np.asarray(bias, np.float64)
    off = off + 2 * F32 * np.abs(y)
    if gelu:
        y = y * 0.5 * torch.erfc(torch.from_numpy(-y / math.sqrt(2.0))).numpy()
        off = 1.13 * off + 4e-7
    if residual is not None:
        y = y + np.asarray(residual, np.float64)
        off = off + 2 * F32 * np.abs(y)
    return y, off + HALF_STEP[dtype] * np.abs(y) + 1e-38


def rotary(x, frequencies, positions, layout="half", factor=1.0, dtype="fp32"):
    """(y, bound): sine and cosine of an angle in fp32 turns (pi 2^-24 of rounding, two steps of the functions), two products and a sum."""
    x = np.asarray(x, np.float64)
    y, off = x.copy(), np.zeros_like(x)
    n = len(frequencies)
    angle = np.asarray(positions, np.float64)[:, None] * np.asarray(frequencies, np.float64)
    cos, sin = np.cos(angle)[:, None], np.sin(angle)[:, None]
    a, b = (slice(0, n), slice(n, 2 * n)) if layout == "half" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    xa, xb = x[..., a], x[..., b]
    y[..., a] = (xa * cos - xb * sin) * factor
    y[..., b] = (xb * cos + xa * sin) * factor
    off[..., a] = off[..., b] = (np.abs(xa) + np.abs(xb)) * abs(factor) * 2.0 ** -21
    off[..., : 2 * n] += HALF_STEP[dtype] * np.abs(y[..., : 2 * n]) + 1e-38
    return y, off


def visible(m, n, first, left, right, prefix, doc_q, doc_k):
    j, d = np.arange(n)[None], np.arange(n)[None] - (first + np.arange(m))[:, None]
    see = ((d >= -left) | (left < 0)) & ((d <= right) | (right < 0)) | (j < prefix)
    if doc_q is not None:
        see = see & (np.asarray(doc_q)[:, None] == np.asarray(doc_k)[None]) & (np.asarray(doc_k)[None] >= 0)
    return see


def attention(q, k, v, cu_q, cu_k, scale=None, cap=0.0, left=-1, right=-1, prefix=None, q_first=None, doc_q=None, doc_k=None,
              slopes=None, bias=None, dtype="fp32"):
    """(out, lse, bound on out, bound on lse); rows of no sequence are NaN.

    A score is off by at most `e`: its fp32 sum of D products (D + 4 half steps of the sum of magnitudes), the tanh (2^-20 of the cap) and what is
    added to it.  Weights are then off by a factor within exp(+-2 e), each sum of n terms by n half steps, and bf16 rounds the weights
    to half a step, as it does the result."""
    q, k, v = (np.asarray(t, np.float64) for t in (q, k, v))
    heads, width, share = q.shape[1], q.shape[2], q.shape[1] // k.shape[1]
    scale = 1.0 / math.sqrt(width) if scale is None else scale
    out, obound = np.full(q.shape, np.nan), np.zeros(q.shape)
    lse, lbound = np.full(q.shape[:2], np.nan), np.zeros(q.shape[:2])
    for b in range(len(cu_q) - 1):
        (a0, a1), (c0, c1) = cu_q[b: b + 2], cu_k[b: b + 2]
        m, n = a1 - a0, c1 - c0
        first = n - m if q_first is None else int(q_first[b])
        see = visible(m, n, first, left, right, 0 if prefix is None else int(prefix[b]), None if doc_q is None else doc_q[a0:a1],
                      None if doc_k is None else doc_k[c0:c1])
        d = np.arange(n)[None] - (first + np.arange(m))[:, None]
        for h in range(heads):
            kk, vv = k[c0:c1, h // share].copy(), v[c0:c1, h // share].copy()
            unseen = ~see.any(0)                            # keys that nobody sees may hold anything
            kk[unseen], vv[unseen] = 0.0, 0.0
            s = q[a0:a1, h] @ kk.T * scale
            e = (width + 4) * F32 * (np.abs(q[a0:a1, h]) @ np.abs(kk).T) * abs(scale)
            if cap > 0:
                s = cap * np.tanh(s / cap)
                e = e + cap * 2.0 ** -20
            if slopes is not None:
                s = s - float(slopes[h]) * np.abs(d)
                e = e + 4 * F32 * (np.abs(s) + float(abs(slopes[h])) * np.abs(d))
            if bias is not None:
                reach = bias.shape[1] // 2
                t = np.asarray(bias[h], np.float64)[np.clip(d, -reach, reach) + reach]
                s = s + t
                e = e + 4 * F32 * (np.abs(s) + np.where(np.isfinite(t), np.abs(t), 0.0))
            s = np.where(see, s, -np.inf)
            e = np.where(np.isfinite(s), e + 8 * F32 * np.abs(np.where(np.isfinite(s), s, 0.0)), 0.0)
            top = s.max(1, initial=-np.inf)
            some = np.isfinite(top)
            p = np.exp(np.where(some[:, None], s - np.where(some, top, 0.0)[:, None], -np.inf))
            total = p.sum(1)
            w = p / np.where(some, total, 1.0)[:, None]
            far = e.max(1, initial=0.0) + (n + 16) * F32
            out[a0:a1, h] = w @ vv
            lse[a0:a1, h] = np.where(some, np.where(some, top, 0.0) + np.log(np.where(some, total, 1.0)), -np.inf)
            reach_v = w @ np.abs(vv)
            step = HALF_STEP[dtype]
            obound[a0:a1, h] = reach_v * (2 * far[:, None] + (step if dtype == "bf16" else 0.0)) + step * np.abs(out[a0:a1, h]) + 1e-30
            lbound[a0:a1, h] = far + 4 * F32 * np.abs(np.where(some, lse[a0:a1, h], 0.0)) + 1e-30
    return out, lse, obound, lbound
