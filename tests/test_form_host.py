"""What Students.set_attention_form keeps alive, on the host: the library and the streams are stand-ins."""
import gc
import weakref

import pytest
import torch

from paper_2408_12526_amd import sp


class Library:
    def __getattr__(self, name):
        return lambda *a: 0


class Stream:
    cuda_stream = 0


@pytest.fixture
def students(monkeypatch):
    st = sp.Students.__new__(sp.Students)
    st.cfg, st.device, st.handle = sp.make_config(2, 1, 128, 2, 256, 30, 16, 3), torch.device("cpu"), 0
    st._ws = st._form = None
    st._form_streams, st._form_captured, st._kept_forms = set(), False, []
    st.capturing, st.recorded = False, []
    monkeypatch.setattr(sp, "_lib", Library())
    monkeypatch.setattr(sp, "_capturing", lambda stream: st.capturing, raising=False)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: st.recorded.append((t.data_ptr(), s)))
    return st


def form():
    return dict(rotary_frequencies=torch.ones(32, dtype=torch.float64), slopes=torch.ones(2, 2), bias=torch.ones(2, 2, 9))


CALLS = {
    "forward": lambda st, s: st.sp_forward_profiled(torch.zeros(4), torch.zeros(3), 2, 2, logits_out=torch.zeros(2, 3), workspace=torch.zeros(1), stream=s),
    "partial": lambda st, s: st.sp_forward_partial(torch.zeros(4), torch.zeros(3), 2, 2, 1, workspace=torch.zeros(1), stream=s),
}


@pytest.mark.parametrize("call", CALLS)
def test_a_replaced_form_waits_for_the_streams_of_its_calls(students, call):
    one, two, idle = Stream(), Stream(), Stream()
    CALLS[call](students, idle)                             # (no form yet)
    old = form()
    at, refs = {t.data_ptr() for t in old.values()}, [weakref.ref(t) for t in old.values()]
    students.set_attention_form(**old)
    for s in (one, two, one):
        CALLS[call](students, s)
    assert students.recorded == []
    new = form()
    students.set_attention_form(**new)
    assert len(students.recorded) == 6 and set(students.recorded) == {(a, s) for a in at for s in (one, two)}
    del old
    gc.collect()
    assert all(r() is None for r in refs)                   # (the allocator's part from here on)
    students.set_attention_form()
    CALLS[call](students, one)
    students.set_attention_form()
    assert len(students.recorded) == 6                      # (no call read the second form)


@pytest.mark.parametrize("call", CALLS)
def test_a_captured_form_stays(students, call):
    old = form()
    refs = [weakref.ref(t) for t in old.values()]
    students.set_attention_form(**old)
    students.capturing = True
    CALLS[call](students, Stream())
    students.capturing = False
    CALLS[call](students, Stream())
    for f in (form(), {}, form()):
        students.set_attention_form(**f)
    del old, f
    gc.collect()
    assert all(r() is not None for r in refs) and len(students._kept_forms) == 1


def test_an_unknown_layout_is_a_value_error(students):
    for more in ({}, form()):
        with pytest.raises(ValueError, match="rotary_layout"):
            students.set_attention_form(rotary_layout="other", **more)
    assert students._form is None


@pytest.mark.parametrize("window", [(1 << 32, 3), (3, (1 << 31)), (1.5, 2), (None, 2)])
def test_windows_that_do_not_fit_are_refused(students, window):
    """They would lose their upper bits: 2^32 keys to the left would be none."""
    with pytest.raises(ValueError, match="window"):
        students.set_attention_form(window=window)
    for good in (((1 << 31) - 1, -1), (-(1 << 40), 0)):
        students.set_attention_form(window=good)
