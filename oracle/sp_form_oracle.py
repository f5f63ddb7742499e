"""The K-student forward with a form of attention (sp_set_attention_form), in numpy and 64 bits; independent of the library.

Weights are the canonical blob's tensors by name, [in][out] matrices."""
from __future__ import annotations

import math

import numpy as np
import torch

from . import sp_ops_oracle as ops


class Exact:
    """No rounding: activations and operands of the projections as they are."""

    def act(self, t):
        return t

    operand = act


class Rounded:
    """Every stored activation off by up to half a step of bf16, every operand of a projection by up to half a step of its type, at random:
    what the path's types may do to the result, whatever its kernels.  kind: "bf16", "fp8" (e4m3 of 16 times the value) or "int8"."""

    def __init__(self, rng, kind):
        self.rng, self.kind = rng, kind

    def _u(self, t):
        return self.rng.uniform(-1.0, 1.0, t.shape)

    def act(self, t):
        return t * (1.0 + 2.0 ** -8 * self._u(t))

    def operand(self, t):
        if self.kind == "fp8":
            return t + np.maximum(2.0 ** -4 * np.abs(t), 2.0 ** -14) * self._u(t)
        if self.kind == "int8":
            return t + np.abs(t).max(-1, keepdims=True) / 254.0 * self._u(t)
        return t


def _layernorm(x, g, b, eps):
    d = x - x.mean(-1, keepdims=True)
    return d / np.sqrt((d * d).mean(-1, keepdims=True) + eps) * g + b


def _gelu(x):
    return x * 0.5 * torch.erfc(torch.from_numpy(-x / math.sqrt(2.0))).numpy()


def layer(x, w, p, heads, eps, cu, student=0, frequencies=None, layout="half", factor=1.0, cap=0.0, window=(-1, -1), slopes=None, bias=None,
          rounding=Exact()):
    """One layer of rows x [tokens, hidden]; w: the student's tensors, p: the layer's prefix, slopes and bias of all students."""
    n, H = x.shape
    xo, act, operand = rounding.operand(x), rounding.act, rounding.operand
    q, k, v = (act((xo @ w[p + "W" + c] + w[p + "b" + c]).reshape(n, heads, H // heads)) for c in "qkv")
    if frequencies is not None:
        pos = np.concatenate([np.arange(b - a) for a, b in zip(cu[:-1], cu[1:])])
        q, k = (act(ops.rotary(t, frequencies, pos, layout, factor)[0]) for t in (q, k))
    att = act(ops.attention(q, k, v, cu, cu, cap=cap, left=window[0], right=window[1], slopes=None if slopes is None else slopes[student],
                        bias=None if bias is None else bias[student])[0].reshape(n, H))
    x1 = act(_layernorm(act(x + operand(att) @ w[p + "Wo"] + w[p + "bo"]), w[p + "ln1_g"], w[p + "ln1_b"], eps))
    g = act(_gelu(operand(x1) @ w[p + "W1"] + w[p + "b1"]))
    return act(_layernorm(act(x1 + operand(g) @ w[p + "W2"] + w[p + "b2"]), w[p + "ln2_g"], w[p + "ln2_b"], eps))


def forward(students, heads, layers, eps, ids, cu, k_active, rounding=Exact(), **form):
    """Logits [batch, classes]: the sum over the first k_active students' heads."""
    pos = np.concatenate([np.arange(b - a) for a, b in zip(cu[:-1], cu[1:])])
    total = 0.0
    for m in range(k_active):
        w = {n: np.asarray(t, np.float64) for n, t in students[m].items()}
        x = rounding.act(_layernorm(w["tok_emb"][ids] + w["pos_emb"][pos], w["emb_ln_g"], w["emb_ln_b"], eps))
        for l in range(layers):
            x = layer(x, w, f"l{l}.", heads, eps, cu, student=m, rounding=rounding, **form)
        total = total + np.tanh(x[cu[:-1]] @ w["Wp"] + w["bp"]) @ w["Wc"] + w["bc"]
    return total


def tolerance(want, kind, *args, draws=2, **form):
    """Three times the largest change of the logits in `draws` forwards whose roundings are off at random (see Rounded)."""
    return 3.0 * max(np.abs(forward(*args, rounding=Rounded(np.random.default_rng(100 + i), kind), **form) - want).max() for i in range(draws))
