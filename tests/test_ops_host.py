"""The operators' C entries on the host: what they refuse before anything reaches a GPU, the frequencies, and the oracle's own pins."""
import ctypes as C
import gc
import math
import weakref

import numpy as np
import pytest
import torch

from oracle import sp_ops_oracle as oracle
from paper_2408_12526_amd import ops, sp

LIB = sp.raw_lib()
EINVAL, ESHAPE, ENOMEM = -1, -2, -4
P = 1 << 20                                                # an aligned address that is never read: every call here is refused


def linear(**k):
    a = dict(x=P, x_row=64, dtype=0, tokens=4, width_in=64, w=2 * P, w_row=64, ws=3 * P, width_out=8, bias=None, epilogue=0, residual=None,
             residual_row=0, out=4 * P, out_row=8, work=5 * P, bytes=1 << 20) | k
    return LIB.sp_linear_int8(*a.values(), None)


@pytest.mark.parametrize("change,code", [
    (dict(x=None), EINVAL), (dict(w=None), EINVAL), (dict(ws=None), EINVAL), (dict(out=None), EINVAL), (dict(work=None), EINVAL),
    (dict(dtype=2), EINVAL), (dict(dtype=-1), EINVAL), (dict(epilogue=3), EINVAL), (dict(epilogue=2), EINVAL), (dict(residual=P * 6), EINVAL),
    (dict(x=P + 2), EINVAL), (dict(w=P + 8), EINVAL), (dict(work=P + 128), EINVAL), (dict(bias=P + 1), EINVAL), (dict(out=P), EINVAL),
    (dict(epilogue=2, residual=4 * P, residual_row=9, out_row=8), EINVAL),
    (dict(tokens=-1), ESHAPE), (dict(width_in=0), ESHAPE), (dict(width_in=131073, w_row=131088), ESHAPE), (dict(width_out=0), ESHAPE),
    (dict(w_row=60), ESHAPE), (dict(w_row=72), ESHAPE), (dict(w_row=48), ESHAPE), (dict(out_row=7), ESHAPE), (dict(x_row=-64), ESHAPE),
    (dict(tokens=1 << 26), ESHAPE), (dict(w_row=(1 << 20) + 16), ESHAPE),
    (dict(bytes=0), ENOMEM), (dict(bytes=4 * 128 + 15), ENOMEM),
])
def test_linear_refuses(change, code):
    assert linear(**change) == code


def test_linear_without_tokens():
    assert linear(tokens=0) == 0
    assert LIB.sp_linear_int8_workspace_bytes(0, 64) == 0
    assert LIB.sp_linear_int8_workspace_bytes(4, 64) == 4 * 128 + 16


def test_quantize_refuses():
    call = LIB.sp_quantize_int8
    assert call(None, 8, 0, 2, 8, P, 8, P, None) == EINVAL
    assert call(P, 8, 1, 2, 8, None, 8, P, None) == EINVAL
    assert call(P, 8, 2, 2, 8, P, 8, P, None) == EINVAL
    assert call(P, 8, 0, 2, 0, P, 8, P, None) == ESHAPE
    assert call(P, 8, 0, 2, 8, P, 7, P, None) == ESHAPE
    assert call(P, 8, 0, 0, 8, P, 8, P, None) == 0
    assert call(P, 8, 0, 1 << 26, 8, P, 8, P, None) == ESHAPE


@pytest.mark.parametrize("width", [(1 << 31) - 1, (1 << 31) - 17, (1 << 31) - 1024, (1 << 31) - 2048])
def test_quantize_refuses_rows_whose_units_pass_32_bits(width):
    """64 units of 16 elements behind the row's end are still formed in 32 bits."""
    assert LIB.sp_quantize_int8(P, width, 1, 1, width, P, width, P, None) == ESHAPE


def rotary(**k):
    a = dict(x=P, xt=128, xh=64, out=2 * P, ot=128, oh=64, dtype=0, tokens=4, heads=2, width=64, dim=64, layout=0, f=3 * P, factor=1.0,
             pos=4 * P, cu=None, batch=0) | k
    return LIB.sp_rotary(*a.values(), None)


@pytest.mark.parametrize("change,code", [
    (dict(x=None), EINVAL), (dict(out=None), EINVAL), (dict(f=None), EINVAL), (dict(pos=None), EINVAL), (dict(cu=P), EINVAL), (dict(dtype=2), EINVAL),
    (dict(layout=2), EINVAL), (dict(f=P + 4), EINVAL), (dict(pos=P + 2), EINVAL), (dict(x=P + 2), EINVAL), (dict(out=P, ot=256), EINVAL),
    (dict(tokens=-1), ESHAPE), (dict(heads=0), ESHAPE), (dict(dim=63), ESHAPE), (dict(dim=66), ESHAPE), (dict(dim=0), ESHAPE), (dict(oh=63), ESHAPE),
    (dict(ot=64), ESHAPE), (dict(xt=-1), ESHAPE), (dict(pos=None, cu=P, batch=-1), ESHAPE), (dict(tokens=1 << 30), ESHAPE),
])
def test_rotary_refuses(change, code):
    assert rotary(**change) == code


def attend(**k):
    a = ops.sp_attention_args(q=P, k=2 * P, v=3 * P, out=4 * P, q_token=128, q_head=64, k_token=128, k_head=64, v_token=128, v_head=64, out_token=128,
                              out_head=64, cu_q=5 * P, cu_k=6 * P, dtype=1, batch=2, heads=2, kv_heads=2, width=64, total_q=8, total_k=8, max_q=8, max_k=8,
                              scale=1.0, left=-1, right=-1)
    for n, v in k.items():
        setattr(a, n, v)
    return LIB.sp_attention(C.addressof(a), None, 0, None)


@pytest.mark.parametrize("change,code", [
    (dict(q=None), EINVAL), (dict(k=None), EINVAL), (dict(v=None), EINVAL), (dict(out=None), EINVAL), (dict(cu_q=None), EINVAL), (dict(cu_k=None), EINVAL),
    (dict(dtype=2), EINVAL), (dict(q=P + 8), EINVAL), (dict(lse=P + 2), EINVAL), (dict(doc_q=P), EINVAL), (dict(scale=math.nan), EINVAL),
    (dict(cap=math.inf), EINVAL), (dict(reach=-1), EINVAL), (dict(q_token=132), EINVAL), (dict(out=P), EINVAL), (dict(out=2 * P), EINVAL),
    (dict(heads=3), ESHAPE), (dict(kv_heads=0), ESHAPE), (dict(width=4), ESHAPE), (dict(width=136), ESHAPE), (dict(width=60), ESHAPE),
    (dict(batch=-1), ESHAPE), (dict(total_q=-1), ESHAPE), (dict(max_k=-1), ESHAPE), (dict(out_head=0), ESHAPE), (dict(out_token=64), ESHAPE), (dict(k_token=-128), ESHAPE),
    (dict(v_token=(1 << 23) + 8), ESHAPE), (dict(total_q=(1 << 29) + 1), ESHAPE), (dict(total_q=1 << 29, heads=4), ESHAPE), (dict(batch=65536), ESHAPE),
    (dict(batch=65535, heads=128, kv_heads=128), ESHAPE), (dict(bias=7 * P, reach=1 << 20, heads=1024, kv_heads=1024), ESHAPE),
])
def test_attention_refuses(change, code):
    assert attend(**change) == code


def test_attention_of_nothing():
    assert attend(total_q=0, q=None, out=None, cu_q=None) == 0
    assert attend(batch=0) == 0
    assert LIB.sp_attention(None, None, 0, None) == EINVAL
    assert LIB.sp_attention_workspace_bytes(None) == 0


def test_arrays_of_nothing_may_be_null():
    """Empty tensors have no address."""
    assert rotary(tokens=0, pos=None, x=None, out=None) == 0 and rotary(tokens=0, pos=None, x=None, out=None, xt=256) == 0
    assert attend(total_q=0, q=None, out=None, doc_k=P) == 0
    assert attend(total_k=0, max_k=0, k=None, v=None, doc_q=P, batch=0) == 0
    assert attend(doc_k=P) == EINVAL and attend(total_k=0, doc_k=P) == EINVAL and attend(total_q=0, doc_q=P) == EINVAL


def test_no_cpu_path():
    x = torch.ones(4, 32)
    with pytest.raises(ValueError):
        ops.quantize_int8(x)
    with pytest.raises(ValueError):
        ops.rotary(torch.ones(4, 2, 64), torch.ones(32, dtype=torch.float64), positions=torch.zeros(4, dtype=torch.int32))
    with pytest.raises(ValueError):
        ops.attention(*[torch.ones(4, 2, 64)] * 3, torch.tensor([0, 4], dtype=torch.int32), 4)


def test_attention_holds_its_workspace_through_the_call(monkeypatch):
    """Between a split call's two launches nobody else may be given the memory: its tensor lives until the call has returned."""
    made, seen = [], []
    empty = torch.empty

    def remember(*a, **k):
        t = empty(*a, **k)
        made.append((weakref.ref(t), t.data_ptr()))
        return t

    class Library:
        @staticmethod
        def sp_attention_workspace_bytes(args):
            return 4096

        @staticmethod
        def sp_attention(args, workspace, size, stream):
            gc.collect()
            seen.extend(r() is not None for r, at in made if at == workspace and r() is not None and r().numel() >= size == 4096)
            return 0

    monkeypatch.setattr(ops, "_home", lambda *a: 0)
    monkeypatch.setattr(ops, "_call", lambda dev, fn, *a: fn(*a, None))
    monkeypatch.setattr(ops, "_lib", Library)
    monkeypatch.setattr(ops.torch, "empty", remember)
    q, cu = torch.ones(4, 2, 64), torch.tensor([0, 4], dtype=torch.int32)
    ops.attention(q, q.clone(), q.clone(), cu, 4)
    assert seen == [True]


def test_sizes_that_leave_32_bits_are_refused(monkeypatch):
    """Views of one element as 2^32 + 5 rows or columns: the library would see five of them."""
    monkeypatch.setattr(ops, "_home", lambda *a: 0)
    monkeypatch.setattr(ops, "_call", lambda *a: pytest.fail("the call was made"))
    monkeypatch.setattr(torch.Tensor, "new_empty", lambda t, shape: t[:1, :1].expand(shape))
    monkeypatch.setattr(ops.torch, "empty", lambda *shape, **k: torch.zeros(1, dtype=k["dtype"]).expand(shape if len(shape) > 1 else 1))
    far = (1 << 32) + 5
    one, code = torch.ones(1, 16), torch.ones(1, 16, dtype=torch.int8)
    with pytest.raises(ValueError):
        ops.quantize_int8(one.expand(far, 16))
    with pytest.raises(ValueError):
        ops.linear_int8(one.expand(far, 16), code, torch.ones(1))
    x = torch.ones(1, 1, 64)
    with pytest.raises(ValueError):
        ops.rotary(x.expand(far, 1, 64), torch.ones(32, dtype=torch.float64), cu_seqlens=torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError):
        ops.rotary(x.expand(1, far, 64), torch.ones(32, dtype=torch.float64), cu_seqlens=torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError):
        ops.attention(x.expand(far, 1, 64), x, x, torch.zeros(2, dtype=torch.int32), 1, torch.zeros(2, dtype=torch.int32), 1)


# ---- frequencies ------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dim", [2, 4, 40, 64, 128])
@pytest.mark.parametrize("factor", [1.0, 4.0, 32.0])
def test_frequencies(dim, factor):
    i = np.arange(dim // 2)
    plain = 10000.0 ** (-2.0 * i / dim)
    f, m = ops.rotary_frequencies(dim)
    assert np.abs(f / plain - 1).max() < 1e-15 * 8 and m == 1.0
    f, m = ops.rotary_frequencies(dim, scaling="linear", factor=factor)
    assert np.abs(f / (plain / factor) - 1).max() < 1e-14 and m == 1.0
    f, m = ops.rotary_frequencies(dim, scaling="parts", factor=factor, trained=2048)
    turns = 2048 * plain / (2 * math.pi)
    assert np.abs(f[turns >= 32] / plain[turns >= 32] - 1).max(initial=0.0) < 1e-14
    assert np.abs(f[turns <= 1] * factor / plain[turns <= 1] - 1).max(initial=0.0) < 1e-14
    mid = (turns > 1) & (turns < 32)
    assert ((f[mid] <= plain[mid] * (1 + 1e-14)) & (f[mid] >= plain[mid] / factor * (1 - 1e-14))).all()
    assert abs(m - (1 + 0.1 * math.log(factor))) < 1e-6
    if dim >= 4:
        f, m = ops.rotary_frequencies(dim, scaling="ntk", factor=factor)
        assert abs(f[0] - 1) < 1e-14                        # the fastest pair stays, the slowest is stretched by the factor
        assert abs(f[-1] * factor / plain[-1] - 1) < 1e-12 and m == 1.0


def test_frequencies_refuse():
    for bad in (dict(dim=3), dict(dim=0), dict(dim=2, scaling="ntk", factor=2), dict(dim=4, factor=0.5), dict(dim=4, base=1.0), dict(dim=4, base=math.inf),
                dict(dim=4, scaling="parts", factor=2.0, trained=0), dict(dim=4, factor=math.nan), dict(dim=4, scaling="other")):
        with pytest.raises((sp.SpError, ValueError)):
            ops.rotary_frequencies(**bad)


# ---- the oracle against library routines ------------------------------------------------------------------------

def test_oracle_attention_is_softmax_attention():
    rng = np.random.default_rng(0)
    q, k, v = (rng.standard_normal((9, 2, 16)) for _ in range(3))
    out, lse, _, _ = oracle.attention(q, k, v, [0, 9], [0, 9], right=0)
    t = [torch.from_numpy(x).transpose(0, 1)[None] for x in (q, k, v)]
    want = torch.nn.functional.scaled_dot_product_attention(*t, is_causal=True)[0].transpose(0, 1).numpy()
    assert np.abs(out - want).max() < 1e-12
    s = (t[0][0] @ t[1][0].transpose(1, 2)).numpy() / 4
    s = np.where(np.tril(np.ones((9, 9), bool)), s, -np.inf)
    assert np.abs(lse.T - torch.logsumexp(torch.from_numpy(s), -1).numpy()).max() < 1e-12


def test_oracle_linear_is_a_product():
    rng = np.random.default_rng(1)
    x, w = rng.standard_normal((5, 64)).astype(np.float32), rng.standard_normal((7, 64)).astype(np.float32)
    c, s = oracle.quantize(x)
    assert np.abs(c).max() == 127 and np.abs(c * s[:, None] - x).max() <= (0.5 * s * (1 + 1e-5)).max()
    cw, sw = oracle.quantize(w)
    y, bound = oracle.linear_int8(x, cw, sw, gelu=True)
    want = torch.nn.functional.gelu(torch.from_numpy((c * s[:, None]) @ (cw * sw[:, None]).T)).numpy()
    assert np.abs(y - want).max() < 1e-12 and (bound > 0).all()
