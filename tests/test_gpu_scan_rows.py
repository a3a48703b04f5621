"""Rows of the gated linear recurrence: gaps between those that it writes, where its memory begins, and row pointers as they may come."""
import pytest
import torch

from test_gpu_scan import TYPES, check, dgn, make  # noqa: F401

pytestmark = pytest.mark.gpu


def test_kept_states_at_an_address_aligned_to_their_elements(dgn):  # noqa: F811
    i = make([100, 0, 77], 33, 1, "sigmoid", "bf16")
    b = check(dgn, i, 33, 1, "sigmoid", "bf16", "kept")
    store = torch.zeros(b._carry.numel() + 4, dtype=torch.uint8, device="cuda")
    carry, want = store[4:], [t.clone() for t in (b.y, b.final, b.dx, b.dgate, b.dh0)]
    for t in (b.y, b.final, b.dx, b.dgate, b.dh0):
        t.zero_()
    assert carry.data_ptr() % 8 == 4
    rc = dgn.dgn_scan_forward(b._d, i["x"], i["gate"], i["rowptr"], i["h0"], b.y, b.final, carry, b._scratch, b._scratch_bytes)
    assert rc == 0
    rc = dgn.dgn_scan_backward(b._d, i["x"], i["gate"], i["rowptr"], i["h0"], carry, i["dy"], i["dfinal"], b.dx, b.dgate, b.dh0,
                               b._scratch, b._scratch_bytes)
    assert rc == 0 and all(torch.equal(s, t) for s, t in zip(want, (b.y, b.final, b.dx, b.dgate, b.dh0)))


@pytest.mark.parametrize("heads,group", [(33, 1), (3, 8)])
def test_inputs_and_outputs_as_columns_of_one_matrix(dgn, heads, group):  # noqa: F811
    """Rows that lie between each other's do not overlap; dh0 in h0's place; one token's y in x's place."""
    c = heads * group
    i = make([100, 0, 377], heads, group, "sigmoid", "bf16")
    b = check(dgn, i, heads, group, "sigmoid", "bf16", "columns")
    n, wide = i["x"].shape[0], 4 * c + 2 * heads + 7
    all_of = torch.full((n, wide), 3.0, dtype=torch.bfloat16, device="cuda")
    x, y, dy, dx = (all_of[:, 1 + k * c:1 + (k + 1) * c] for k in range(4))
    gate, dgate = (all_of[:, 2 + 4 * c + k * heads:2 + 4 * c + (k + 1) * heads] for k in range(2))
    x.copy_(i["x"]), gate.copy_(i["gate"]), dy.copy_(i["dy"])
    d = dgn.dgn_scan_desc(n, 3, c, group, dgn.DGN_BF16, dgn.DGN_GATE_SIGMOID, wide, wide, wide, wide, wide, wide)
    states = i["h0"].clone()
    at = lambda t: t.data_ptr()  # noqa: E731
    rc = dgn.dgn_scan_forward(d, at(x), at(gate), i["rowptr"], states, at(y), b.final, b._carry, b._scratch, b._scratch_bytes)
    assert rc == 0
    rc = dgn.dgn_scan_backward(d, at(x), at(gate), i["rowptr"], states, b._carry, at(dy), i["dfinal"], at(dx), at(dgate), states,
                               b._scratch, b._scratch_bytes)
    assert rc == 0
    for got, want in [(y, b.y), (dx, b.dx), (dgate, b.dgate), (states, b.dh0), (x, i["x"]), (gate, i["gate"]), (dy, i["dy"])]:
        assert torch.equal(got, want)
    rest = torch.ones(wide, dtype=torch.bool)
    rest[1:1 + 4 * c] = rest[2 + 4 * c:2 + 4 * c + 2 * heads] = False
    assert (all_of[:, rest.cuda()] == 3.0).all()
    s = dgn.ScanStepBuffers(n, n, c, gate_group=group, kind="sigmoid")
    pool = torch.randn(n, c, device="cuda")
    again, into = pool.clone(), i["x"].clone()
    s.step(i["x"], i["gate"], None, pool)
    assert dgn.dgn_scan_step(s._d, n, into, i["gate"], None, again, again, into) == 0
    assert torch.equal(into, s.y) and torch.equal(again, pool)


def test_outputs_as_inputs_are_refused(dgn):  # noqa: F811
    i = make([12, 8], 12, 1, "decay", "bf16")
    b = dgn.ScanBuffers(20, 2, 12, kind="decay", train=True)
    b.forward(i["x"], i["gate"], i["rowptr"], h0=i["h0"])
    for bad in [dict(x=b.y), dict(gate=b.y)]:
        with pytest.raises(dgn.DgnError):
            b.forward(**{**dict(x=i["x"], gate=i["gate"], seq_rowptr=i["rowptr"]), **bad})
    for bad in [dict(x=b.dx), dict(dy=b.dx), dict(gate=b.dgate), dict(dy=b.dgate)]:
        with pytest.raises(dgn.DgnError):
            b.backward(**{**dict(x=i["x"], gate=i["gate"], seq_rowptr=i["rowptr"], dy=i["dy"]), **bad})
    b.backward(i["x"], i["gate"], i["rowptr"], b.y, h0=i["h0"], dfinal=b.final)         # outputs of forward are inputs like others
