"""Students with a form of attention (sp_set_attention_form) and students quantised in 8-bit integers (SP_DTYPE_INT8), against
64-bit oracles.  Needs an MI355X.

Tolerances: fp32 1e-3 absolute on logits, as for the plain students; else three times what roundings of the path's types, off at random at the
places where it rounds, make of the oracle's logits (sp_form_oracle.tolerance): with queries and keys this large the softmax is so
sharp that half a step of bf16 in a query of 30 turns a score by a tenth, whatever the kernels.  An 8-bit projection checked on the input that the forward left in the workspace carries only the roundings of the operator itself."""
import numpy as np
import pytest
import torch

from oracle import sp_form_oracle, sp_ops_oracle
from paper_2408_12526_amd import ops, sp, synth

pytestmark = pytest.mark.gpu


def shape_of(dtype, hidden=128, K=2, ffn=256, layers=2):
    return synth.StudentShape(K=K, layers=layers, hidden=hidden, heads=hidden // 64, ffn=ffn, vocab=300, max_pos=320, classes=3, dtype=dtype)


def make(shape, lengths, seed=3):
    rng = np.random.default_rng(seed)
    blob = synth.make_weights(rng, shape, std=0.05, ln_random=True, qk_std=0.2)
    lengths = np.array(lengths, np.int32)
    return blob, synth.make_ids(rng, int(lengths.sum()), shape.vocab), sp.sp_pack(lengths), int(lengths.max())


def students_of(blob, shape, tokens=0, layers=None, first_only=False):
    """What the oracle consumes: the weights as the group keeps them, rounded to bf16, or in large calls of quantised students as 8-bit codes
    times their scales (fp8 with a form of attention: all but the output projection; behind the last layer's attention the first tokens alone
    are computed, in bf16, unless the group says otherwise)."""
    if shape.dtype == "fp32":
        return [synth.student_views(blob, shape, m) for m in range(shape.K)]
    w = torch.from_numpy(blob).bfloat16().float().numpy()
    out = [synth.student_views(w, shape, m) for m in range(shape.K)]
    if shape.dtype in ("fp8", "int8") and (tokens + 255) // 256 * 256 >= 2048:
        for m, views in synth.iter_views(blob, shape):
            for name, x in views.items():
                kind = name.split(".")[-1]
                if layers is not None and not name.startswith(layers):
                    continue
                if first_only and name.startswith(f"l{shape.layers - 1}.") and kind in ("Wo", "W1", "W2"):
                    continue
                if kind not in ("Wq", "Wk", "Wv", "Wo", "W1", "W2") or (shape.dtype == "fp8" and kind == "Wo"):
                    continue
                if shape.dtype == "int8":
                    codes, scales = sp_ops_oracle.quantize(np.ascontiguousarray(x.T))
                    out[m][name] = (codes * scales[:, None]).T
                else:
                    t = torch.from_numpy(np.ascontiguousarray(x))
                    scale = t.abs().amax(0) / 448.0
                    out[m][name] = ((t / scale).to(torch.float8_e4m3fn).double() * scale.double()).numpy()
    return out


def form_of(shape, which):
    rng = np.random.default_rng(8)
    f, factor = ops.rotary_frequencies(32 if which == "part" else 64, base=500.0, scaling="parts" if which == "all" else "none", factor=2.0 if which == "all" else 1.0, trained=64)
    form = {}
    if which in ("rotary", "part", "all"):
        form.update(frequencies=f, layout="interleaved" if which == "part" else "half", factor=factor)
    if which in ("cap", "all"):
        form.update(cap=2.0)
    if which in ("window", "all"):
        form.update(window=(9, 4))
    if which in ("slopes",):
        form.update(slopes=(rng.random((shape.K, shape.heads)) * 0.2).astype(np.float32))
    if which in ("table", "all"):
        form.update(bias=rng.standard_normal((shape.K, shape.heads, 31)).astype(np.float32))
    return form


def set_form(st, form):
    d = {n: torch.from_numpy(v).cuda() if isinstance(v, np.ndarray) else v for n, v in form.items()}
    if "frequencies" in d:
        d["rotary_frequencies"], d["rotary_layout"], d["rotary_factor"] = d.pop("frequencies"), d.pop("layout"), d.pop("factor")
    st.set_attention_form(**d)


LENGTHS = {"few": [5, 1, 33], "some": [5, 1, 96, 33, 64, 200, 70, 129], "many": [200, 1, 129] + [40, 77, 64, 9, 32] * 8}


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp8", "int8"])
@pytest.mark.parametrize("which", ["rotary", "part", "cap", "window", "slopes", "table", "all"])
@pytest.mark.parametrize("size", LENGTHS)
def test_forms(dtype, which, size):
    shape = shape_of(dtype, hidden=256 if dtype == "fp8" else 128, ffn=512)
    blob, ids, cu, most = make(shape, LENGTHS[size])
    form = form_of(shape, which)
    whole = which in ("window", "all")                      # (the last layer for all tokens, else for the first ones only)
    st = sp.Students(sp.config_from_shape(shape, last_layer_all_tokens=whole), blob)
    d_ids, d_cu = torch.from_numpy(ids).cuda(), torch.from_numpy(cu).cuda()
    plain = st.sp_forward(d_ids, d_cu, most, shape.K).clone()
    set_form(st, form)
    for k in (shape.K, 1) if size == "some" else (shape.K,):
        got = st.sp_forward(d_ids, d_cu, most, k).double().cpu().numpy()
        args = students_of(blob, shape, len(ids), first_only=not whole), shape.heads, shape.layers, shape.ln_eps, ids, cu, k
        want = sp_form_oracle.forward(*args, **form)
        tol = 1e-3 if dtype == "fp32" else sp_form_oracle.tolerance(want, dtype if len(ids) > 1792 else "bf16", *args, **form)
        assert np.abs(got - want).max() <= tol
    assert np.abs(got - plain.double().cpu().numpy()).max() > 0
    set_form(st, {})
    assert torch.equal(st.sp_forward(d_ids, d_cu, most, shape.K), plain)


@pytest.mark.parametrize("dtype", ["bf16", "int8"])
def test_form_in_two_groups_and_in_a_graph(dtype):
    """A call large enough for two groups of students on two streams, captured and replayed: the bits of one stream."""
    shape = shape_of(dtype, hidden=512, K=4, ffn=512)
    blob, ids, cu, most = make(shape, [256, 100, 300] * 24)
    assert len(ids) >= 8192 and len(ids) * shape.K * shape.hidden >= 20 << 20
    form = form_of(shape, "all")
    d_ids, d_cu = torch.from_numpy(ids).cuda(), torch.from_numpy(cu).cuda()
    one = sp.Students(sp.config_from_shape(shape, single_stream=True), blob)
    two = sp.Students(sp.config_from_shape(shape), blob)
    set_form(one, form)
    set_form(two, form)
    want = one.sp_forward(d_ids, d_cu, most, shape.K)
    out = two.sp_forward(d_ids, d_cu, most, shape.K)
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        two.sp_forward(d_ids, d_cu, most, shape.K, logits_out=out)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def over(st, form):
    """Replaces the form by nothing and writes NaN over whatever memory that gave back."""
    st.set_attention_form()
    sizes = {n: v.nbytes for n, v in form.items() if isinstance(v, np.ndarray)}
    return [torch.full((size // 4,), float("nan"), device="cuda") for size in sizes.values() for _ in range(64)]


@pytest.mark.parametrize("size", LENGTHS)
def test_a_captured_call_keeps_its_form(size):
    shape = shape_of("bf16")
    blob, ids, cu, most = make(shape, LENGTHS[size])
    form = form_of(shape, "all")
    st = sp.Students(sp.config_from_shape(shape), blob)
    d_ids, d_cu = torch.from_numpy(ids).cuda(), torch.from_numpy(cu).cuda()
    set_form(st, form)
    want = st.sp_forward(d_ids, d_cu, most, shape.K).clone()
    out = torch.empty_like(want)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        st.sp_forward(d_ids, d_cu, most, shape.K, logits_out=out)
    filled = over(st, form)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        st.sp_forward(d_ids, d_cu, most, shape.K)
    assert len(filled) == 2 * 64


def test_a_call_on_another_stream_keeps_its_form():
    """The form is replaced, and its memory given out again, while a call that was issued with it still waits on its stream."""
    shape = shape_of("bf16")
    blob, ids, cu, most = make(shape, LENGTHS["some"])
    form = form_of(shape, "all")
    st = sp.Students(sp.config_from_shape(shape), blob)
    d_ids, d_cu = torch.from_numpy(ids).cuda(), torch.from_numpy(cu).cuda()
    set_form(st, form)
    want = st.sp_forward(d_ids, d_cu, most, shape.K).clone()
    a = torch.randn(8192, 8192, device="cuda")
    ws = torch.empty_like(st.workspace(len(ids), len(cu) - 1))
    out = torch.empty_like(want)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for _ in range(8):                                  # (tens of milliseconds in front of the call)
            a = a @ a
    st.sp_forward(d_ids, d_cu, most, shape.K, logits_out=out, workspace=ws, stream=side)
    filled = over(st, form)
    torch.cuda.synchronize()
    assert torch.equal(out, want) and len(filled) == 2 * 64


@pytest.mark.parametrize("hidden,ffn", [(128, 384), (256, 512), (384, 640)])
@pytest.mark.parametrize("with_form", [False, True])
def test_int8_projections_stage_by_stage(hidden, ffn, with_form):
    """Each 8-bit projection on the input that the forward left in the workspace, rounded like the operator's results."""
    shape = shape_of("int8", hidden=hidden, ffn=ffn, layers=1)
    blob, ids, cu, most = make(shape, [200, 1, 129] + [64] * 33)
    T, B, K, H = int(cu[-1]), len(cu) - 1, shape.K, hidden
    assert T >= 2048
    st = sp.Students(sp.config_from_shape(shape, last_layer_all_tokens=True), blob)
    if with_form:
        set_form(st, form_of(shape, "cap"))
    d_ids, d_cu = torch.from_numpy(ids).cuda(), torch.from_numpy(cu).cuda()
    x = st.read_activation(st.sp_forward_partial(d_ids, d_cu, most, K, 0), "x", T, B, K)
    ws = st.sp_forward_partial(d_ids, d_cu, most, K, 1)
    a = {n: st.read_activation(ws, n, T, B, K) for n in ("qkv", "att", "x1", "g", "x")}
    for m, w in synth.iter_views(blob, shape):
        cols = {n: sp_ops_oracle.quantize(np.ascontiguousarray(w["l0." + n].T)) for n in ("Wq", "Wk", "Wv", "Wo", "W1", "W2")}
        for i, n in enumerate("qkv"):
            want, bound = sp_ops_oracle.linear_int8(x[m], *cols["W" + n], w["l0.b" + n], dtype="bf16")
            assert (np.abs(a["qkv"][m][:, i * H: (i + 1) * H] - want) <= bound).all(), n
        want, bound = sp_ops_oracle.linear_int8(a["x1"][m], *cols["W1"], w["l0.b1"], gelu=True, dtype="bf16")
        assert (np.abs(a["g"][m] - want) <= bound).all()
        # behind the other two stands a LayerNorm: its input is rounded to bf16 (half a step of rows of up to `top`), divided by their spread
        for got, src, n, res, ln in ((a["x1"][m], a["att"][m], "Wo", x[m], "ln1"), (a["x"][m], a["g"][m], "W2", a["x1"][m], "ln2")):
            u, bound = sp_ops_oracle.linear_int8(src, *cols[n], w["l0.bo" if n == "Wo" else "l0.b2"], residual=res, dtype="bf16")
            want = sp_form_oracle._layernorm(u, w[f"l0.{ln}_g"], w[f"l0.{ln}_b"], shape.ln_eps)
            spread = u.std(1, keepdims=True)
            # d LN = g (du - mean du - n mean(n du)) / spread with |n| = |want - b| / |g|: three times the largest input error of the row
            off = 3 * np.abs(w[f"l0.{ln}_g"]).max() * bound.max(1, keepdims=True) * (1 + np.abs((u - u.mean(1, keepdims=True)) / spread)) / spread
            assert (np.abs(got - want) <= off + 2.0 ** -8 * np.abs(want) + 1e-5).all(), n


@pytest.mark.parametrize("hidden,K", [(128, 3), (256, 2), (768, 2)])
@pytest.mark.parametrize("last_all", [False, True])
def test_int8_students(hidden, K, last_all):
    """Whole forwards, on both sides of the line of 2048 rows, first-token last layer (in bf16) and whole one."""
    shape = shape_of("int8", hidden=hidden, K=K, ffn=2 * hidden)
    for lengths in ([5, 1, 33], [64, 200, 3] * 4, [64, 200, 3, 31] * 9):
        blob, ids, cu, most = make(shape, lengths)
        st = sp.Students(sp.config_from_shape(shape, last_layer_all_tokens=last_all), blob)
        got = st.sp_forward(torch.from_numpy(ids).cuda(), torch.from_numpy(cu).cuda(), most, K).double().cpu().numpy()
        args = students_of(blob, shape, len(ids), ("l0.", "l1.") if last_all else ("l0.",)), shape.heads, shape.layers, shape.ln_eps, ids, cu, K
        want = sp_form_oracle.forward(*args)
        assert np.abs(got - want).max() <= sp_form_oracle.tolerance(want, "int8" if len(ids) > 1792 else "bf16", *args)


def test_form_refusals():
    shape = shape_of("bf16")
    blob, ids, cu, most = make(shape, [5, 9])
    st = sp.Students(sp.config_from_shape(shape), blob)
    f = torch.ones(32, dtype=torch.float64, device="cuda")
    for bad in (dict(rotary_frequencies=f.float()), dict(rotary_frequencies=torch.ones(33, dtype=torch.float64, device="cuda")), dict(rotary_frequencies=f.cpu()),
                dict(cap=float("inf")), dict(slopes=torch.ones(2, 3, device="cuda")), dict(bias=torch.ones(2, 2, 4, device="cuda")),
                dict(bias=torch.ones(1, 2, 5, device="cuda")), dict(rotary_frequencies=f, rotary_factor=float("nan"))):
        with pytest.raises((ValueError, sp.SpError)):
            st.set_attention_form(**bad)
    d_ids, d_cu = torch.from_numpy(ids).cuda(), torch.from_numpy(cu).cuda()
    assert torch.isfinite(st.sp_forward(d_ids, d_cu, most, 2)).all()
