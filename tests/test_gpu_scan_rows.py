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


@pytest.mark.parametrize("heads,group", [(66, 1), (1, 1), (3, 8), (2, 96), (2, 300)])
@pytest.mark.parametrize("lens", [[77], [300, 0, 41], [900, 1]])
def test_outputs_with_gaps(dgn, heads, group, lens):  # noqa: F811
    """Rows of y, dx and dgate further apart than they are wide, by odd numbers: the same values (which `check` holds to the plain
    form), and what lies between is not touched."""
    c = heads * group
    for kind, dtype in [("decay", "bf16"), ("sigmoid", "f32"), ("sigmoid", "f16")]:
        i = make(lens, heads, group, kind, dtype, pad=(3, 5))
        b = check(dgn, i, heads, group, kind, dtype, "gaps")
        n, seqs = i["x"].shape[0], len(lens)
        stores = {name: torch.full((n, w + gap), 7.0, dtype=TYPES[dtype], device="cuda")
                  for name, w, gap in (("y", c, 3), ("dx", c, 7), ("dgate", heads, 1))}
        d = dgn.dgn_scan_desc(n, seqs, c, group, b._d.dtype, b._d.gate_kind, 0, 0, c + 3, 0, c + 7, heads + 1)
        final, dh0, carry = torch.zeros_like(b.final), torch.zeros_like(b.dh0), torch.zeros_like(b._carry)
        rc = dgn.dgn_scan_forward(d, i["x"], i["gate"], i["rowptr"], i["h0"], stores["y"][:, 1:].data_ptr(), final, carry, b._scratch,
                                  b._scratch_bytes)
        assert rc == 0
        rc = dgn.dgn_scan_backward(d, i["x"], i["gate"], i["rowptr"], i["h0"], carry, i["dy"], i["dfinal"],
                                   stores["dx"][:, 1:].data_ptr(), stores["dgate"][:, 1:].data_ptr(), dh0, b._scratch, b._scratch_bytes)
        assert rc == 0 and torch.equal(final, b.final) and torch.equal(dh0, b.dh0)
        for name, w in (("y", c), ("dx", c), ("dgate", heads)):
            assert torch.equal(stores[name][:, 1:1 + w], getattr(b, name)), name       # (rows outside the sequences: 7 in both)
            assert (stores[name][:, 0] == 7.0).all() and (stores[name][:, 1 + w:] == 7.0).all(), name
        s = dgn.ScanStepBuffers(n, n, c, gate_group=group, kind=kind, dtype=TYPES[dtype])
        pool, again = (torch.ones(n, c, device="cuda") for _ in range(2))
        y = torch.full((n, c + 5), 7.0, dtype=TYPES[dtype], device="cuda")
        s.step(i["x"], i["gate"], None, pool)
        d = dgn.dgn_scan_desc(n, 0, c, group, b._d.dtype, b._d.gate_kind, 0, 0, c + 5, 0, 0, 0)
        assert dgn.dgn_scan_step(d, n, i["x"], i["gate"], None, again, again, y[:, 2:].data_ptr()) == 0
        assert torch.equal(again.isnan(), pool.isnan()) and torch.equal(again.nan_to_num(), pool.nan_to_num())
        assert torch.equal(y[:, 2:2 + c].isnan(), s.y.isnan()) and torch.equal(y[:, 2:2 + c].nan_to_num(), s.y.nan_to_num())
        assert (y[:, :2] == 7.0).all() and (y[:, 2 + c:] == 7.0).all()


def test_every_row_past_32_bits(dgn):  # noqa: F811
    """x, gate, y and the gradients with rows so far apart that the last ones lie more than 2^32 bytes behind the first."""
    rows, stride, c = 300, 2**23, 30
    i = make([rows - 50, 50], c, 1, "sigmoid", "bf16")
    b = check(dgn, i, c, 1, "sigmoid", "bf16", "far")
    far = {}
    for name in ("x", "gate", "dy", "y", "dx", "dgate"):
        store = torch.empty((rows - 1) * stride + 64, dtype=torch.bfloat16, device="cuda")
        far[name] = store.as_strided((rows, c), (stride, 1))
        if name in i:
            far[name].copy_(i[name])
    d = dgn.dgn_scan_desc(rows, 2, c, 1, dgn.DGN_BF16, dgn.DGN_GATE_SIGMOID, *[stride] * 6)
    at = {name: t.data_ptr() for name, t in far.items()}
    final, dh0 = torch.zeros_like(b.final), torch.zeros_like(b.dh0)
    rc = dgn.dgn_scan_forward(d, at["x"], at["gate"], i["rowptr"], i["h0"], at["y"], final, b._carry, b._scratch, b._scratch_bytes)
    assert rc == 0
    rc = dgn.dgn_scan_backward(d, at["x"], at["gate"], i["rowptr"], i["h0"], b._carry, at["dy"], i["dfinal"], at["dx"], at["dgate"], dh0,
                               b._scratch, b._scratch_bytes)
    assert rc == 0
    for name in ("y", "dx", "dgate"):
        assert torch.equal(far[name], getattr(b, name)), name
    assert torch.equal(final, b.final) and torch.equal(dh0, b.dh0)


def test_states_of_a_pool_past_32_bits(dgn):  # noqa: F811
    """One token for rows whose states lie more than 2^32 bytes into the pool."""
    slots, c = 300_000, 4100
    i = make([1] * 6, c, 1, "sigmoid", "f32")
    pool = torch.empty(slots, c, device="cuda")
    slot = torch.tensor([0, slots - 1, 262_144, -1, 131_072, 299_000], dtype=torch.int32, device="cuda")
    live = slot >= 0
    pool[slot[live].long()] = i["h0"][live]
    small, s = dgn.ScanStepBuffers(6, 6, c, dtype=torch.float32), dgn.ScanStepBuffers(6, slots, c, dtype=torch.float32)
    states = i["h0"].clone()
    small.step(i["x"], i["gate"], torch.where(live, torch.arange(6, device="cuda", dtype=torch.int32), -1), states)
    s.step(i["x"], i["gate"], slot, pool)
    assert torch.equal(s.y, small.y) and torch.equal(pool[slot[live].long()], states[live])


@pytest.mark.parametrize("heads,group", [(40, 1), (2, 130)])
@pytest.mark.parametrize("n", [60, 700])
def test_row_pointers_outside_the_rows_and_out_of_order(dgn, heads, group, n):  # noqa: F811
    """Pointers outside 0 .. n count as 0 and n.  Those that do not ascend give values of no meaning, but nothing else is touched: the
    buffers have guards before and after them."""
    c, seqs, guard = heads * group, 3, 4096
    i = make([n // 3, 0, n - n // 3], heads, group, "sigmoid", "f32")
    desc = dgn.dgn_scan_desc(n, seqs, c, group, dgn.DGN_F32, dgn.DGN_GATE_SIGMOID)
    _, nb, cb = dgn.dgn_scan_workspace(desc)
    shapes = dict(y=(n, c), dx=(n, c), dgate=(n, heads), final=(seqs, c), dh0=(seqs, c), carry=(cb // 4,), scratch=(nb // 4,))

    def call(rowptr):
        stores = {k: torch.full((torch.Size(s).numel() + 2 * guard,), 7.0, device="cuda") for k, s in shapes.items()}
        at = {k: t[guard:].data_ptr() for k, t in stores.items()}
        rowptr = torch.tensor(rowptr, device="cuda")
        rc = dgn.dgn_scan_forward(desc, i["x"], i["gate"], rowptr, i["h0"], at["y"], at["final"], at["carry"], at["scratch"], nb)
        assert rc == 0
        rc = dgn.dgn_scan_backward(desc, i["x"], i["gate"], rowptr, i["h0"], at["carry"], i["dy"], i["dfinal"], at["dx"], at["dgate"],
                                   at["dh0"], at["scratch"], nb)
        assert rc == 0
        for name, t in stores.items():
            assert (t[:guard] == 7.0).all() and (t[-guard:] == 7.0).all(), (name, rowptr.tolist())
        return {k: stores[k][guard:-guard] for k in ("y", "dx", "dgate", "final", "dh0")}
    third = n // 3
    want, got = call([0, third, third, n]), call([-2**40, third, third, n + 2**40])
    assert all(torch.equal(want[k], got[k]) for k in want)
    for wild in ([0, n, third, n], [n, third, third, 0], [5, n + 9, -3, n], [third, 0, n, third], [2**62, -2**62, 2**62, -2**62]):
        call(wild)


@pytest.mark.parametrize("heads,group,kind,dtype", [(2, 1, "sigmoid", "bf16"), (1, 24, "decay", "f32")])
def test_more_strips_than_stay_in_registers(dgn, heads, group, kind, dtype):  # noqa: F811
    """More than 1 024 strips: the launch between goes over the links twice.  Pieces of 17 and of fewer strips, forward and backward."""
    i = make([20011, 0, 45000, 1000], heads, group, kind, dtype)
    check(dgn, i, heads, group, kind, dtype, "many strips")
