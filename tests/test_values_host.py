"""Host-side checks of the operators on tensor values that need no GPU: what the library refuses before any device work."""
import ctypes

import numpy as np
import pytest
import torch

import values_oracle as vo


@pytest.fixture(scope="module")
def d():
    import paper_1707_08265_amd as d
    return d


def desc(d, **kw):
    base = dict(num_tokens=10, num_seqs=2, num_channels=12, gate_group=3, dtype=d.DGN_BF16, gate_kind=d.DGN_GATE_DECAY)
    return d.dgn_scan_desc(**{**base, **kw})


def test_scan_description_is_checked(d):
    ok = d.dgn_scan_workspace(desc(d))
    assert ok[0] == 0 and ok[2] >= 12 * 4 and ok[1] % 8 == 0
    for bad, code in [(dict(num_tokens=-1), d.DGN_ERR_INVALID_ARG), (dict(num_seqs=-1), d.DGN_ERR_INVALID_ARG),
                      (dict(num_channels=-1), d.DGN_ERR_INVALID_ARG), (dict(gate_group=0), d.DGN_ERR_INVALID_ARG),
                      (dict(gate_group=5), d.DGN_ERR_INVALID_ARG), (dict(dtype=3), d.DGN_ERR_INVALID_ARG),
                      (dict(dtype=-1), d.DGN_ERR_INVALID_ARG), (dict(gate_kind=2), d.DGN_ERR_INVALID_ARG),
                      (dict(x_stride=11), d.DGN_ERR_INVALID_ARG), (dict(gate_stride=3), d.DGN_ERR_INVALID_ARG),
                      (dict(dgate_stride=-4), d.DGN_ERR_INVALID_ARG), (dict(num_tokens=2**31 - 1), d.DGN_ERR_TOO_LARGE),
                      (dict(num_seqs=2**31), d.DGN_ERR_TOO_LARGE), (dict(num_channels=3 * 2**31), d.DGN_ERR_TOO_LARGE),
                      (dict(y_stride=2**41), d.DGN_ERR_TOO_LARGE)]:
        assert d.dgn_scan_workspace(desc(d, **bad))[0] == code, bad
        assert d.dgn_scan_step(desc(d, **bad), 4, 64, 64, None, 64, 64, 64, stream=0) == code, bad
    assert d.dgn_scan_workspace(None)[0] == d.DGN_ERR_NULL_PTR
    assert d.dgn_scan_workspace(desc(d, x_stride=12, gate_stride=4, dgate_stride=4))[0] == 0


def test_scan_calls_refuse_bad_pointers(d):
    m = desc(d)
    _, sb, _ = d.dgn_scan_workspace(m)
    good = dict(x=64, gate=64, rowptr=64, h0=64, y=64, final=64, carry=64, scratch=64, nb=sb)

    def forward(**kw):
        a = {**good, **kw}
        return d.dgn_scan_forward(m, a["x"], a["gate"], a["rowptr"], a["h0"], a["y"], a["final"], a["carry"], a["scratch"],
                                  a["nb"], stream=0)

    def backward(**kw):
        a = {**good, "dy": 64, "dfinal": 64, "dx": 64, "dgate": 64, "dh0": 64, **kw}
        return d.dgn_scan_backward(m, a["x"], a["gate"], a["rowptr"], a["h0"], a["carry"], a["dy"], a["dfinal"], a["dx"],
                                   a["dgate"], a["dh0"], a["scratch"], a["nb"], stream=0)
    for name in ("x", "gate", "rowptr", "y"):
        assert forward(**{name: 0}) == d.DGN_ERR_NULL_PTR, name
    for name in ("x", "gate", "rowptr", "carry", "dy", "dx", "dgate"):
        assert backward(**{name: 0}) == d.DGN_ERR_NULL_PTR, name
    for name, off in [("x", 1), ("gate", 1), ("y", 1), ("h0", 2), ("final", 2), ("rowptr", 4), ("carry", 2), ("scratch", 4)]:
        assert forward(**{name: 64 + off}) == d.DGN_ERR_INVALID_ARG, name
    for name, off in [("dy", 1), ("dx", 1), ("dgate", 1), ("dh0", 2), ("dfinal", 2), ("rowptr", 4), ("carry", 2), ("scratch", 4)]:
        assert backward(**{name: 64 + off}) == d.DGN_ERR_INVALID_ARG, name
    if sb:
        assert forward(nb=sb - 1) == d.DGN_ERR_WORKSPACE_TOO_SMALL and backward(nb=sb - 1) == d.DGN_ERR_WORKSPACE_TOO_SMALL
    # nothing to do: no channels, no sequences, no rows
    for empty in (desc(d, num_channels=0), desc(d, num_seqs=0)):
        assert d.dgn_scan_forward(empty, None, None, None, None, None, None, None, None, 0, stream=0) == 0
        assert d.dgn_scan_backward(empty, None, None, None, None, None, None, None, None, None, None, None, 0, stream=0) == 0
    assert d.dgn_scan_step(desc(d, num_tokens=0), 3, None, None, None, None, None, None, stream=0) == 0
    step = lambda slots=None, n=4, x=64, si=64, so=64, y=64: d.dgn_scan_step(m, n, x, 64, slots, si, so, y, stream=0)  # noqa: E731
    assert step(n=-1) == d.DGN_ERR_INVALID_ARG and step(n=2**31) == d.DGN_ERR_TOO_LARGE
    assert step(x=0) == d.DGN_ERR_NULL_PTR and step(y=0) == d.DGN_ERR_NULL_PTR and step(si=0) == d.DGN_ERR_NULL_PTR
    assert step(so=0) == d.DGN_ERR_NULL_PTR and step(slots=66) == d.DGN_ERR_INVALID_ARG and step(y=65) == d.DGN_ERR_INVALID_ARG


def list_desc(d, numel, dtype=None, data=None):
    n = len(numel)
    keep = (np.array(data if data is not None else [256] * n, np.uint64), np.array(numel, np.int64),
            np.array(dtype if dtype is not None else [d.DGN_F32] * n, np.int32))
    out = d.dgn_list_desc(count=n, data=keep[0].ctypes.data, numel=keep[1].ctypes.data, dtype=keep[2].ctypes.data)
    out.keep = keep
    return out


def test_list_description_is_checked(d):
    assert d.dgn_list_workspace(None)[0] == d.DGN_ERR_NULL_PTR
    rc, small = d.dgn_list_workspace(list_desc(d, [5, 0, 7]))
    rc2, large = d.dgn_list_workspace(list_desc(d, [5, 0, 70_000_000]))
    assert rc == rc2 == 0 and 0 < small < large
    assert d.dgn_list_workspace(d.dgn_list_desc(count=0))[0] == 0
    assert d.dgn_list_workspace(d.dgn_list_desc(count=-1))[0] == d.DGN_ERR_INVALID_ARG
    assert d.dgn_list_workspace(d.dgn_list_desc(count=2**31))[0] == d.DGN_ERR_TOO_LARGE
    assert d.dgn_list_workspace(d.dgn_list_desc(count=1))[0] == d.DGN_ERR_NULL_PTR
    for kw, code in [(dict(numel=[-1]), d.DGN_ERR_INVALID_ARG), (dict(numel=[2**45]), d.DGN_ERR_TOO_LARGE),
                     (dict(numel=[2**43] * 9), d.DGN_ERR_TOO_LARGE), (dict(numel=[1], dtype=[7]), d.DGN_ERR_INVALID_ARG),
                     (dict(numel=[1], data=[0]), d.DGN_ERR_NULL_PTR), (dict(numel=[1], data=[258]), d.DGN_ERR_INVALID_ARG),
                     (dict(numel=[1], data=[257], dtype=[d.DGN_BF16]), d.DGN_ERR_INVALID_ARG)]:
        assert d.dgn_list_workspace(list_desc(d, **kw))[0] == code, kw
    one = list_desc(d, [5])
    nb = d.dgn_list_workspace(one)[1]
    assert d.dgn_list_build(one, None, nb, stream=0) == (d.DGN_ERR_NULL_PTR, None)
    assert d.dgn_list_build(one, 256, nb - 1, stream=0)[0] == d.DGN_ERR_WORKSPACE_TOO_SMALL
    assert d.dgn_list_build(one, 260, nb, stream=0)[0] == d.DGN_ERR_INVALID_ARG
    d.dgn_list_destroy(None)


def test_list_calls_refuse_missing_handles(d):
    assert d.dgn_list_norms_workspace(None)[0] == d.DGN_ERR_NULL_PTR
    assert d.dgn_list_norms(None, None, 64, 64, 1 << 20, stream=0) == d.DGN_ERR_NULL_PTR
    assert d.dgn_list_clip(None, None, None, 64, 1.0, stream=0) == d.DGN_ERR_NULL_PTR
    assert d.dgn_list_adam(None, None, None, d.dgn_adam_options(), stream=0) == d.DGN_ERR_NULL_PTR
    assert d.dgn_list_adam(d.dgn_adam_lists(), None, None, d.dgn_adam_options(), stream=0) == d.DGN_ERR_NULL_PTR


def test_structures_have_the_sizes_of_the_header(d):
    assert ctypes.sizeof(d.dgn_scan_desc) == 4 * 8 + 2 * 4 + 6 * 8
    assert ctypes.sizeof(d.dgn_list_desc) == 32 and ctypes.sizeof(d.dgn_reach) == 32
    assert ctypes.sizeof(d.dgn_adam_lists) == 64 and ctypes.sizeof(d.dgn_adam_options) == 5 * 8 + 8 + 3 * 4 + 4


@pytest.mark.parametrize("kind", ["decay", "sigmoid"])
def test_the_plain_recurrence_agrees_with_its_differences(kind):
    """The 64-bit form that the kernels are compared with: its gradients against central differences of its own loss."""
    gen = torch.Generator().manual_seed(3)
    rn = lambda *s: torch.randn(*s, generator=gen, dtype=torch.float64)  # noqa: E731
    rowptr, group = torch.tensor([0, 4, 4, 11]), 2
    x, gate, h0, dy, dfinal = rn(11, 6), rn(11, 3), rn(3, 6), rn(11, 6), rn(3, 6)
    if kind == "decay":
        gate = torch.sigmoid(gate)

    def loss(x, gate, h0):
        r = vo.scan(x, gate, rowptr, kind, group, h0)
        return float((r["y"][0] * dy).sum() + (r["final"][0] * dfinal).sum())
    r = vo.scan(x, gate, rowptr, kind, group, h0, dy, dfinal)
    for i, name in enumerate(("dx", "dgate", "dh0")):
        args = [x, gate, h0]
        way = torch.randn(args[i].shape, generator=gen, dtype=torch.float64)
        up, down = list(args), list(args)
        up[i], down[i] = args[i] + 1e-5 * way, args[i] - 1e-5 * way
        assert abs((loss(*up) - loss(*down)) / 2e-5 - float((r[name][0] * way).sum())) < 1e-7, name
