"""Performance cases of the operators of `paper_2408_12526_amd.ops`: products in 8-bit integers, rotary positions, and
attention with capped scores, distance biases and masks.

A case is one call on tensors that are already on the device.  With `own` false the same operator is computed by elementary
torch operations on padded tensors in 32 bits; with `own` true by the library.  Lengths are quantiles of a named
distribution, so that a case has one total; their order and all values come from the seed.
"""
from __future__ import annotations

import math
from statistics import NormalDist

import numpy as np
import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


# ---- cases ------------------------------------------------------------------------------------------------------

def _linear(name, dtype, tokens, width_in, width_out, epilogue):
    return dict(name=name, op="linear", dtype=dtype, tokens=tokens, width_in=width_in, width_out=width_out, epilogue=epilogue)


def _rotary(name, dtype, tokens, heads, width, dim, layout, scaling="none", factor=1.0, span=512):
    return dict(name=name, op="rotary", dtype=dtype, tokens=tokens, heads=heads, width=width, dim=dim, layout=layout,
                scaling=scaling, factor=factor, span=span)


def _attend(name, dtype, batch, kind, lo, hi, heads, kv_heads, width, queries="all", median=0, cap=0.0, slopes=False, reach=0,
            causal=False, left=-1, right=-1, prefix=0.0, docs=0):
    return dict(name=name, op="attend", dtype=dtype, batch=batch, kind=kind, lo=lo, hi=hi, median=median, heads=heads,
                kv_heads=kv_heads, width=width, queries=queries, cap=cap, slopes=slopes, reach=reach, causal=causal, left=left,
                right=right, prefix=prefix, docs=docs)


def listed():
    return [
        # one row through the query/key/value projection: the first token of a lone request
        _linear("linear_one_row", "bf16", 1, 768, 2304, "bias"),
        # a request of 64 tokens up a BERT-large-width feed-forward layer
        _linear("linear_request", "bf16", 64, 1024, 4096, "gelu"),
        # widths that fill no tile and no load, in 32 bits
        _linear("linear_odd", "fp32", 1999, 1000, 777, "residual"),
        # a burst of 14.7 k tokens down the feed-forward layer
        _linear("linear_burst", "bf16", 14722, 4096, 1024, "residual"),
        # queries and keys of a lone request
        _rotary("rotary_request", "bf16", 64, 24, 64, 64, "half"),
        # an odd number of tokens, part of the head, neighbouring pairs, in 32 bits
        _rotary("rotary_part_fp32", "fp32", 4999, 12, 80, 40, "interleaved", "linear", 4.0, 2048),
        # long documents far into their context, frequencies scaled by parts
        _rotary("rotary_long", "bf16", 65536, 20, 128, 128, "half", "parts", 16.0, 1 << 20),
        # the first token's query of every sequence of a batch of long requests: all that the head of an encoder reads
        _attend("attend_first", "bf16", 64, "uniform", 64, 512, 16, 16, 64, queries="first", reach=128),
        # one new token each against long caches, eight queries to a key head, capped scores
        _attend("attend_last_long", "bf16", 8, "uniform", 1000, 32768, 32, 4, 128, queries="last", cap=30.0),
        # the burst of short requests with a learned bias by distance
        _attend("attend_burst", "bf16", 256, "lognormal", 8, 256, 12, 12, 64, median=48, reach=64),
        # 32 bits, a bias that falls with the distance, both directions
        _attend("attend_fp32", "fp32", 32, "uniform", 16, 301, 8, 8, 64, slopes=True),
        # long packed documents with padding, a window to the left and a prefix that everybody sees, capped scores, shared heads
        _attend("attend_documents", "bf16", 4, "uniform", 4096, 8192, 16, 4, 128, cap=50.0, causal=True, left=2048, prefix=0.02, docs=3),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A call of any of the operators, of any size up to the largest listed one."""
    op = rng.choice(["linear", "linear", "rotary", "attend", "attend", "attend"])
    dtype = "fp32" if rng.random() < 0.25 else "bf16"
    if op == "linear":
        c = _linear("", dtype, _log_int(rng, 1, 14722), _log_int(rng, 64, 4096), _log_int(rng, 64, 4096), rng.choice(["bias", "gelu", "residual"]))
        while work(c)["flops"] > work(listed()[3])["flops"]:
            c["tokens"] = (c["tokens"] + 1) // 2
    elif op == "rotary":
        width = 8 * rng.randint(4, 16)
        dim = width if rng.random() < 0.6 else 2 * rng.randint(4, width // 2)
        scaling = rng.choice(["none", "linear", "ntk", "parts"])
        c = _rotary("", dtype, _log_int(rng, 16, 65536 if dtype == "bf16" else 32768), rng.randint(1, 20), width, dim, rng.choice(["half", "interleaved"]),
                    scaling, 1.0 if scaling == "none" else float(rng.choice([2, 4, 16])), _log_int(rng, 512, 1 << 20))
    else:
        width = rng.choice([64, 64, 128, 8 * rng.randint(4, 16)])
        kv_heads = rng.choice([1, 2, 4, 8, 12])
        heads = kv_heads * rng.choice([1, 1, 2, 4]) if kv_heads <= 4 else kv_heads
        bias = rng.choice(["none", "slopes", "table"])
        how = dict(cap=rng.choice([0.0, 0.0, 20.0, 50.0]), slopes=bias == "slopes", reach=_log_int(rng, 8, 512) if bias == "table" else 0)
        if rng.random() < 0.4:
            hi = _log_int(rng, 64, 32768)
            c = _attend("", dtype, _log_int(rng, 1, max(1, min(256, 262144 // hi))), "uniform", max(1, hi // 16), hi, heads, kv_heads, width,
                        queries=rng.choice(["first", "last"]), **how)
        else:
            hi = _log_int(rng, 16, 4096)
            batch = _log_int(rng, 1, max(1, min(256, (1 << 24) // (hi * hi))))
            causal = rng.random() < 0.4
            left = _log_int(rng, 8, hi) if rng.random() < 0.4 else -1
            right = _log_int(rng, 8, hi) if left >= 0 and not causal else -1
            c = _attend("", dtype, batch, "uniform", max(1, hi // 8), hi, heads, kv_heads, width, causal=causal, left=left, right=right,
                        prefix=rng.choice([0.0, 0.1]) if causal or left >= 0 else 0.0, docs=rng.choice([0, 0, 2, 5]), **how)
    del c["name"]
    return c


# ---- inputs -----------------------------------------------------------------------------------------------------

def _lengths(case):
    """The batch's lengths, ascending: the quantiles of the named distribution."""
    u = (np.arange(case["batch"]) + 0.4) / case["batch"]
    lo, hi = case["lo"], case["hi"]
    if case["kind"] == "uniform":
        n = lo + np.floor(u * (hi - lo + 1))
    else:
        n = np.rint(case["median"] * np.exp(0.6 * np.array([NormalDist().inv_cdf(x) for x in u])))
    return np.clip(n, lo, hi).astype(np.int32)


def _documents(length, docs):
    """Document of every token: `docs` of about the same length, then two per cent of padding that belongs to none."""
    d = np.arange(length) * docs // max(1, length - length // 50)
    return np.where(d < docs, d, -1).astype(np.int32)


def _frequencies(case):
    """Radians per position of every pair (64 bits), and the factor on the rotated values."""
    dim, factor = case["dim"], case["factor"]
    base = 10000.0 * (factor ** (dim / (dim - 2)) if case["scaling"] == "ntk" else 1.0)
    f = base ** (-np.arange(0, dim, 2, dtype=np.float64) / dim)
    if case["scaling"] == "linear":
        f = f / factor
    if case["scaling"] == "parts":      # turns within the 4096 positions of training: 1 and fewer are stretched, 32 and more are not
        keep = np.clip((4096 * f / (2 * math.pi) - 1.0) / 31.0, 0.0, 1.0)
        return f * keep + f / factor * (1.0 - keep), 1.0 + 0.1 * math.log(factor)
    return f, 1.0


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    rng = np.random.default_rng(seed)
    dtype = _TYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    if case["op"] == "linear":
        T, K, N = case["tokens"], case["width_in"], case["width_out"]
        x = normal(T, K)
        x[:, :: max(1, K // 6)] *= 8.0                              # a few wide features, as behind a LayerNorm
        w = normal(N, K) * 0.02
        most = w.abs().amax(1)
        codes = torch.zeros(N, (K + 15) // 16 * 16, dtype=torch.int8, device="cuda")
        codes[:, :K] = torch.round(w / (most / 127.0)[:, None]).to(torch.int8)
        return dict(op="linear", epilogue=case["epilogue"], x=x.to(dtype), codes=codes[:, :K], scale=most / 127.0, bias=normal(N) * 0.02,
                    residual=normal(T, N).to(dtype) if case["epilogue"] == "residual" else None)
    if case["op"] == "rotary":
        f, factor = _frequencies(case)
        n = case["tokens"]
        first = int(rng.integers(0, max(1, case["span"] - n)))
        return dict(op="rotary", layout=case["layout"], factor=factor, x=normal(n, case["heads"], case["width"]).to(dtype),
                    frequencies=torch.from_numpy(f).cuda(),
                    positions=torch.from_numpy(((first + np.arange(n)) % case["span"]).astype(np.int32)).cuda())
    n = rng.permutation(_lengths(case))
    m = n if case["queries"] == "all" else np.ones_like(n)
    cu_k, cu_q = (np.concatenate([[0], np.cumsum(v)]).astype(np.int32) for v in (n, m))
    H, G, D = case["heads"], case["kv_heads"], case["width"]

    def dev(a):
        return torch.from_numpy(np.ascontiguousarray(a)).cuda()

    docs = dev(np.concatenate([_documents(int(v), case["docs"]) for v in n])) if case["docs"] else None
    slopes = bias = None
    if case["slopes"]:
        slopes = dev((2.0 ** (-8.0 * (np.arange(H) + 1) / H)).astype(np.float32))
    if case["reach"]:
        bias = normal(H, 2 * case["reach"] + 1)
    return dict(op="attend", q=normal(int(cu_q[-1]), H, D).to(dtype), k=normal(int(cu_k[-1]), G, D).to(dtype), v=normal(int(cu_k[-1]), G, D).to(dtype),
                cu_q=dev(cu_q), cu_k=dev(cu_k), max_q=int(m.max()), max_k=int(n.max()), cap=case["cap"], causal=case["causal"], left=case["left"],
                right=case["right"], docs=docs, slopes=slopes, bias=bias, prefix=dev((n * case["prefix"]).astype(np.int32)) if case["prefix"] else None,
                q_first=dev(np.zeros(len(n), np.int32)) if case["queries"] == "first" else None)


# ---- one pass ---------------------------------------------------------------------------------------------------

def run(state):
    if own:
        return _library(state)
    return {"linear": _plain_linear, "rotary": _plain_rotary, "attend": _plain_attend}[state["op"]](state)


def _library(s):
    from paper_2408_12526_amd import ops
    if s["op"] == "linear":
        return ops.linear_int8(s["x"], s["codes"], s["scale"], s["bias"], residual=s["residual"], gelu=s["epilogue"] == "gelu")
    if s["op"] == "rotary":
        return ops.rotary(s["x"], s["frequencies"], positions=s["positions"], layout=s["layout"], factor=s["factor"])
    return ops.attention(s["q"], s["k"], s["v"], s["cu_q"], s["max_q"], s["cu_k"], s["max_k"], cap=s["cap"], causal=s["causal"],
                         window=(s["left"], s["right"]), prefix=s["prefix"], q_first=s["q_first"], doc_q=s["docs"], doc_k=s["docs"],
                         slopes=s["slopes"], bias=s["bias"], with_lse=True)


def _plain_linear(s):
    x = s["x"].float()
    most = x.abs().amax(1, keepdim=True)
    c127 = torch.full_like(most, 127.0)                             # (a division by a number may become a product)
    codes = torch.round(x * (c127 / most))
    y = torch.matmul(codes, s["codes"].float().t()) * ((most / c127) * s["scale"]) + s["bias"]
    if s["epilogue"] == "gelu":
        y = 0.5 * y * (1.0 + torch.erf(y * math.sqrt(0.5)))
    if s["epilogue"] == "residual":
        y = y + s["residual"].float()
    return y.to(s["x"].dtype)


def _plain_rotary(s):
    x, half = s["x"].float(), s["frequencies"].numel()
    angle = torch.remainder(s["positions"].double()[:, None] * s["frequencies"], 2.0 * math.pi).float()[:, None]
    cos, sin = angle.cos() * s["factor"], angle.sin() * s["factor"]
    if s["layout"] == "half":
        a, b = x[..., :half], x[..., half: 2 * half]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = x[..., 0: 2 * half: 2], x[..., 1: 2 * half: 2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([turned, x[..., 2 * half:]], -1).to(s["x"].dtype)


def _plain_attend(s):
    """Padded to the longest sequence: scores [sequence][head][query][key]."""
    cu_q, cu_k, M, N = s["cu_q"].long(), s["cu_k"].long(), s["max_q"], s["max_k"]
    (Tq, H, D), G, B = s["q"].shape, s["k"].shape[1], s["cu_q"].numel() - 1
    dev = s["q"].device
    rows, cols = torch.arange(M, device=dev), torch.arange(N, device=dev)
    m, n = cu_q[1:] - cu_q[:-1], cu_k[1:] - cu_k[:-1]
    at_q = (cu_q[:-1, None] + rows).clamp(max=Tq - 1)
    at_k = (cu_k[:-1, None] + cols).clamp(max=s["k"].shape[0] - 1)
    q = s["q"][at_q].float().transpose(1, 2).reshape(B, G, H // G * M, D)
    k = s["k"][at_k].float().permute(0, 2, 3, 1).contiguous()
    v = s["v"][at_k].float().transpose(1, 2).contiguous()
    sc = torch.matmul(q, k).view(B, H, M, N).mul_(1.0 / math.sqrt(D))
    if s["cap"] > 0:
        sc = sc.div_(s["cap"]).tanh_().mul_(s["cap"])
    i = (n - m if s["q_first"] is None else s["q_first"].long())[:, None] + rows
    far = cols - i[:, :, None]                                      # [sequence][query][key]
    if s["slopes"] is not None:
        sc = sc.sub_(s["slopes"][:, None, None] * far.abs()[:, None])
    if s["bias"] is not None:
        reach = s["bias"].shape[1] // 2
        sc = sc.add_(s["bias"][:, far.clamp(-reach, reach) + reach].transpose(0, 1))
    right = 0 if s["causal"] else s["right"]
    seen = torch.ones_like(far, dtype=torch.bool)
    if s["left"] >= 0:
        seen &= far >= -s["left"]
    if right >= 0:
        seen &= far <= right
    if s["prefix"] is not None:
        seen |= cols < s["prefix"].long()[:, None, None]
    seen &= cols < n[:, None, None]
    if s["docs"] is not None:
        dq, dk = s["docs"][at_q][:, :, None], s["docs"][at_k][:, None]
        seen &= (dq == dk) & (dk >= 0)
    sc = sc.masked_fill_(~seen[:, None], -math.inf)
    top = sc.amax(-1, keepdim=True)
    base = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = sc.sub_(base).exp_()
    total = p.sum(-1, keepdim=True)
    lse = (base + total.log()).squeeze(-1)
    out = torch.matmul(p.view(B, G, H // G * M, N), v).view(B, H, M, D) / torch.where(total > 0, total, torch.ones_like(total))
    token = torch.arange(Tq, device=dev)
    b = torch.searchsorted(cu_q[1:].contiguous(), token, right=True)
    r = token - cu_q[b]
    return out[b, :, r].to(s["q"].dtype), lse[b, :, r]


# ---- what a pass cannot do without ------------------------------------------------------------------------------

def _pairs(case):
    """Visible pairs of query and key, of all sequences."""
    total = 0
    for n in _lengths(case).astype(int):
        i = np.arange(n) if case["queries"] == "all" else np.array([0 if case["queries"] == "first" else n - 1])
        right = 0 if case["causal"] else case["right"]
        if not case["docs"]:
            spans = [(0, n)]
        else:
            d = _documents(n, case["docs"])
            spans = [(int((d == x).argmax()), int((d == x).argmax() + (d == x).sum())) for x in range(case["docs"]) if (d == x).any()]
        prefix = int(n * case["prefix"])
        for a, z in spans:
            q = i[(i >= a) & (i < z)]
            lo = np.maximum(a, q - case["left"]) if case["left"] >= 0 else np.full(len(q), a)
            hi = np.minimum(z, q + right + 1) if right >= 0 else np.full(len(q), z)
            total += int((hi - lo).sum() + np.clip(np.minimum(prefix, lo) - a, 0, None).sum() + np.clip(min(prefix, z) - hi, 0, None).sum())
    return total


def work(case):
    size = 4 if case["dtype"] == "fp32" else 2
    if case["op"] == "linear":
        T, K, N = case["tokens"], case["width_in"], case["width_out"]
        return {"bytes": T * K * size + N * K + 8 * N + T * N * size * (2 if case["epilogue"] == "residual" else 1), "flops": 2 * T * K * N}
    if case["op"] == "rotary":
        n = case["tokens"]
        return {"bytes": 2 * n * case["heads"] * case["width"] * size + 4 * n + 4 * case["dim"], "flops": 3 * n * case["heads"] * case["dim"]}
    H, G, D = case["heads"], case["kv_heads"], case["width"]
    keys = int(_lengths(case).sum())
    queries = keys if case["queries"] == "all" else case["batch"]
    return {"bytes": size * D * (2 * queries * H + 2 * keys * G) + 4 * queries * H, "flops": 4 * D * H * _pairs(case)}


# ---- the definition in 64 bits ----------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "linear":
        # codes and scales are defined by single operations in 32 bits; what follows is exact
        x = s["x"].float().cpu().numpy()
        a = np.abs(x).max(1)
        c = np.rint(x * (np.float32(127) / a)[:, None])
        t = torch.from_numpy((a / np.float32(127)).astype(np.float64)).cuda()
        y = torch.from_numpy(c.astype(np.float64)).cuda() @ s["codes"].double().t().contiguous()
        y = y * t[:, None] * s["scale"].double()[None] + s["bias"].double()[None]
        if case["epilogue"] == "gelu":
            y = y * torch.special.ndtr(y)
        if case["epilogue"] == "residual":
            y += s["residual"].double()
        return y
    if case["op"] == "rotary":
        f = s["frequencies"]
        turn = torch.polar(torch.full((), s["factor"], dtype=torch.float64, device="cuda"), s["positions"].double()[:, None] * f[None])[:, None]
        x, d = s["x"].double(), 2 * f.numel()
        z = torch.view_as_complex(x[..., :d].unflatten(-1, (2, -1)).transpose(-1, -2).contiguous() if case["layout"] == "half"
                                  else x[..., :d].unflatten(-1, (-1, 2)).contiguous()) * turn
        r = torch.view_as_real(z)
        x[..., :d] = (r.transpose(-1, -2) if case["layout"] == "half" else r).flatten(-2)
        return x
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    cq, ck = s["cu_q"].tolist(), s["cu_k"].tolist()
    share = case["heads"] // case["kv_heads"]
    right = 0 if case["causal"] else case["right"]
    for b in range(case["batch"]):
        m, n = cq[b + 1] - cq[b], ck[b + 1] - ck[b]
        i = torch.arange(m, device="cuda") + (0 if case["queries"] == "first" else n - m)
        j = torch.arange(n, device="cuda")
        d = j[None] - i[:, None]
        hidden = torch.zeros(m, n, dtype=torch.bool, device="cuda")
        if case["left"] >= 0:
            hidden |= d < -case["left"]
        if right >= 0:
            hidden |= d > right
        if s["prefix"] is not None:
            hidden &= (j >= int(s["prefix"][b]))[None]
        if s["docs"] is not None:
            own_doc = s["docs"][ck[b]: ck[b + 1]]
            hidden |= (own_doc[:, None] != own_doc[None]) | (own_doc < 0)[None]
        for h0 in range(0, case["heads"], share):
            k, v = (s[x][ck[b]: ck[b + 1], h0 // share].double() for x in ("k", "v"))
            for h in range(h0, h0 + share):
                z = s["q"][cq[b]: cq[b + 1], h].double() @ k.t().contiguous() / math.sqrt(case["width"])
                if case["cap"]:
                    z = torch.tanh(z / case["cap"]) * case["cap"]
                if s["slopes"] is not None:
                    z = z - s["slopes"][h].double() * d.abs()
                if s["bias"] is not None:
                    z = z + s["bias"][h].double()[d.clamp(-case["reach"], case["reach"]) + case["reach"]]
                z[hidden] = -math.inf
                e = torch.logsumexp(z, 1)
                lse[cq[b]: cq[b + 1], h] = e
                out[cq[b]: cq[b + 1], h] = torch.nan_to_num(torch.exp(z - e[:, None])) @ v
    return out, lse
