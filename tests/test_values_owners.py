"""What the owners of buffers hand to the library, without a GPU."""
from types import SimpleNamespace

import pytest
import torch

import paper_1707_08265_amd as dgn
from paper_1707_08265_amd import values


def test_a_mask_of_no_words_is_still_a_mask():
    lst = type("Two", (SimpleNamespace,), {"__len__": lambda self: 2})(index=-1, _mem=torch.zeros(64, dtype=torch.uint8))
    r = values._reach(lst, 1, torch.zeros(0, dtype=torch.int64), torch.zeros(2, dtype=torch.int32))
    assert r.num_words == 0 and r.tensor_mask and r.tensor_ids


class Lists:
    """Stand-ins for lists of tensors, and a library that notes what it is called with."""

    def __init__(self, monkeypatch):
        self.calls = []
        note = lambda *a: self.calls.append(a) or 0  # noqa: E731
        for name in ("dgn_list_adam", "dgn_list_clip", "dgn_list_norms"):
            monkeypatch.setattr(values.b._lib, name, note)
        monkeypatch.setattr(values, "_current_device", lambda: 0)
        monkeypatch.setattr(values.b, "_raw_stream", lambda index: 0)

    def make(self, n=8, index=0):
        return [SimpleNamespace(handle=1000 + i, index=index) for i in range(n)]


ADAM = dict(lr=1e-2, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1, step=3)


@pytest.mark.parametrize("closed", range(8))
def test_update_with_a_closed_list_is_refused(monkeypatch, closed):
    """Closed after the owner was made: its handle is no longer the library's.  Before: an optional list is not `in place`."""
    env = Lists(monkeypatch)
    lists = env.make()
    a = values.AdamBuffers(*lists)
    a.step(**ADAM)
    assert len(env.calls) == 1
    lists[closed].handle = None
    with pytest.raises(dgn.DgnError):
        a.step(**ADAM)
    with pytest.raises(dgn.DgnError):
        values.AdamBuffers(*lists)
    assert len(env.calls) == 1


def test_buffers_in_host_memory_are_refused():
    """Kernels would be given host addresses: tensors of the same device as the buffers pass every later check."""
    with pytest.raises(dgn.DgnError):
        dgn.ScanBuffers(20, 2, 12, device="cpu")
    with pytest.raises(dgn.DgnError):
        dgn.ScanBuffers(20, 2, 12, train=True, device="cpu")
    with pytest.raises(dgn.DgnError):
        dgn.ScanStepBuffers(4, 8, 12, device="cpu")


@pytest.mark.parametrize("other", range(1, 8))
def test_lists_of_another_device_are_refused(monkeypatch, other):
    env = Lists(monkeypatch)
    lists = env.make()
    lists[other].index = 1
    with pytest.raises(dgn.DgnError):
        values.AdamBuffers(*lists)
    norms = values.GradientBuffers.__new__(values.GradientBuffers)
    norms.grads, norms.num_sets, norms.norms = lists[0], 1, torch.zeros(1)
    norms.clip(lists[0], 1.0)
    with pytest.raises(dgn.DgnError):
        norms.clip(lists[other], 1.0)
    assert len(env.calls) == 1


def test_calls_away_from_the_buffers_device_are_refused(monkeypatch):
    """Kernels run on the current device's stream, which has to be that of the memory."""
    env = Lists(monkeypatch)
    a = values.AdamBuffers(*env.make())
    a.step(**ADAM)
    monkeypatch.setattr(values, "_current_device", lambda: 1)
    with pytest.raises(dgn.DgnError):
        a.step(**ADAM)
    assert len(env.calls) == 1


def test_a_call_keeps_the_strides_that_it_was_given(monkeypatch):
    """The library reads a call's description without Python's lock: the next call must not write to it."""
    with monkeypatch.context() as m:
        m.setattr(values, "_need", lambda ok, where: None)                  # (owners of host buffers are refused)
        s, t = dgn.ScanBuffers(20, 2, 12, kind="decay", train=True, device="cpu"), dgn.ScanStepBuffers(20, 2, 12, device="cpu")
    seen = []
    for name in ("dgn_scan_forward", "dgn_scan_backward", "dgn_scan_step"):
        monkeypatch.setattr(values.b._lib, name, lambda d, *a: seen.append(d._obj) or 0)
    monkeypatch.setattr(values, "_current_device", lambda: -1)
    monkeypatch.setattr(values.b, "_raw_stream", lambda index: 0)
    ptr, pool = torch.tensor([0, 7, 20]), torch.zeros(2, 12)
    wide = torch.zeros(20, 40, dtype=torch.bfloat16)
    want = []
    for a, c, e in [(40, 40, 40), (12, 40, 40), (12, 12, 40), (12, 12, 12), (40, 12, 12)]:
        cut = lambda step: wide[:, 3:15] if step == 40 else wide[:, 3:15].contiguous()  # noqa: E731
        s.forward(cut(a), cut(c), ptr)
        s.backward(cut(c), cut(a), ptr, cut(e))
        t.step(cut(a), cut(e), None, pool)
        want += [(a, c, None), (c, a, e), (a, e, None)]
    got = [(d.x_stride, d.gate_stride, d.dy_stride) for d in seen]
    assert len(got) == len(want)
    for g, w in zip(got, want):
        assert g[:2] == w[:2] and w[2] in (None, g[2])


@pytest.mark.parametrize("bad", [[64], [None], [[1.0]], [torch.zeros(3), 64]])
def test_lists_of_what_is_no_tensor_are_refused(bad):
    with pytest.raises(dgn.DgnError):
        dgn.TensorList(bad)
