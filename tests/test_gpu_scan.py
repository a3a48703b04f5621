"""Gated linear recurrence on the GPU against its plain form in 64 bits (bounds: values_oracle)."""
import pytest
import torch

import values_oracle as vo

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def dgn():
    assert torch.cuda.is_available(), "these tests need the GPU"
    import paper_1707_08265_amd as d
    return d


def make(lens, heads, group, kind, dtype, seed=0, pad=(0, 0), states=True):
    """Inputs on the GPU; pad: rows before the first and after the last sequence (NaN in them)."""
    gen = torch.Generator().manual_seed(seed)
    n, c, s = sum(lens), heads * group, len(lens)
    rn = lambda *shape: torch.randn(*shape, generator=gen)  # noqa: E731
    gate = rn(n, heads) * 1.5 + 2.0
    gate = gate if kind == "sigmoid" else torch.sigmoid(gate)

    def rows(t):
        full = torch.full((pad[0] + n + pad[1], t.shape[1]), float("nan"))
        full[pad[0]:pad[0] + n] = t
        return full.to(TYPES[dtype]).cuda()
    rowptr = torch.tensor([pad[0]] + [pad[0] + sum(lens[:i + 1]) for i in range(s)])
    return dict(x=rows(rn(n, c)), gate=rows(gate), dy=rows(rn(n, c)), rowptr=rowptr.cuda(),
                h0=rn(s, c).cuda() if states else None, dfinal=rn(s, c).cuda() if states else None)


def check(dgn, i, heads, group, kind, dtype, what, train=True):
    n, seqs = i["x"].shape[0], i["rowptr"].numel() - 1
    print(f"scan {what}: {n} rows, {seqs} sequences, {heads} x {group}, {kind}, {dtype}", flush=True)
    b = dgn.ScanBuffers(n, seqs, heads * group, gate_group=group, kind=kind, dtype=TYPES[dtype], train=train)
    names = ["y"] + (["dx", "dgate"] if train else [])
    for name in names:
        getattr(b, name).fill_(7.0)
    b.forward(i["x"], i["gate"], i["rowptr"], h0=i["h0"])
    if train:
        b.backward(i["x"], i["gate"], i["rowptr"], i["dy"], h0=i["h0"], dfinal=i["dfinal"])
    torch.cuda.synchronize()
    want = vo.scan(i["x"], i["gate"], i["rowptr"], kind, group, i["h0"], i["dy"] if train else None, i["dfinal"])
    first, last = int(i["rowptr"][0]), int(i["rowptr"][-1])
    for name, (value, error) in want.items():
        got = getattr(b, name)
        if name in names:
            assert (got[:first] == 7.0).all() and (got[last:] == 7.0).all(), f"{what}: {name} outside the sequences"
            got, value, error = got[first:last], value[first:last], error[first:last]
        vo.within(got, value, error, f"{what}: {name}")
    return b


LENGTHS = {"one": [1], "two": [2], "none": [0], "tile": [128], "past": [129], "short": [127], "mixed": [0, 127, 1, 0, 0, 128, 129, 0],
           "ones": [1] * 300, "long": [1291], "pair": [700, 0, 3, 517], "many": [5, 0, 16, 17, 1, 33] * 20}


@pytest.mark.parametrize("lens", sorted(LENGTHS))
@pytest.mark.parametrize("kind", ["decay", "sigmoid"])
def test_lengths(dgn, kind, lens):
    for dtype in TYPES:
        check(dgn, make(LENGTHS[lens], 70, 1, kind, dtype), 70, 1, kind, dtype, lens)


@pytest.mark.parametrize("heads,group", [(1, 1), (2, 1), (127, 1), (128, 1), (129, 1), (330, 1), (1, 2), (5, 3), (3, 8), (33, 4),
                                         (2, 64), (1, 65), (3, 96), (1, 128), (2, 128), (1, 130), (2, 200), (1, 257), (3, 300)])
def test_layouts(dgn, heads, group):
    for kind, dtype in [("decay", "bf16"), ("sigmoid", "f32"), ("sigmoid", "f16")]:
        check(dgn, make([150, 0, 77], heads, group, kind, dtype, seed=heads), heads, group, kind, dtype, "layout")


@pytest.mark.parametrize("states", [False, True])
@pytest.mark.parametrize("train", [False, True])
def test_states_and_room_for_more_rows(dgn, states, train):
    for pad in [(0, 0), (3, 200), (130, 1)]:
        i = make([5, 0, 260], 40, 1, "sigmoid", "bf16", pad=pad, states=states)
        check(dgn, i, 40, 1, "sigmoid", "bf16", f"pad {pad}", train)


def test_rows_with_gaps_and_odd_addresses(dgn):
    for dtype in TYPES:
        i = make([300, 41], 66, 1, "sigmoid", dtype)
        for name in ("x", "gate", "dy"):
            wide = torch.full((341, 66 + 5), float("nan"), dtype=TYPES[dtype], device="cuda")
            wide[:, 3:69] = i[name]
            i[name] = wide[:, 3:69]
        check(dgn, i, 66, 1, "sigmoid", dtype, "gaps")


def test_gates_at_their_limits(dgn):
    """Gates of 0, 1 and the infinities; states beyond a reset do not come back."""
    inf = float("inf")
    for kind, values in [("decay", [0.0, 1.0, -0.5, 0.999]), ("sigmoid", [-inf, inf, 100.0, -100.0])]:
        i = make([200], 64, 1, kind, "f32")
        i["gate"][:, 3] = torch.tensor(values, device="cuda").repeat(50)
        i["gate"][50:60, 7] = values[0]
        check(dgn, i, 64, 1, kind, "f32", "limits")


def test_what_is_no_number_stays_in_its_sequence_and_channel(dgn):
    for bad in (float("nan"), float("inf")):
        i = make([150, 300, 0, 40], 65, 1, "sigmoid", "bf16")
        clean = check(dgn, i, 65, 1, "sigmoid", "bf16", "clean")
        want = {n: getattr(clean, n).clone() for n in ("y", "final", "dx", "dgate", "dh0")}
        i["x"][150 + 70, 5] = bad
        i["dy"][150 + 70, 9] = bad
        b = dgn.ScanBuffers(490, 4, 65, kind="sigmoid", train=True)
        b.forward(i["x"], i["gate"], i["rowptr"], h0=i["h0"])
        b.backward(i["x"], i["gate"], i["rowptr"], i["dy"], h0=i["h0"], dfinal=i["dfinal"])
        for name, hit in [("y", 5), ("dgate", 5), ("dx", 9), ("dgate", 9)]:
            assert not getattr(b, name)[150:450, hit].isfinite().all(), (name, bad)
        for name, value in want.items():
            got = getattr(b, name).clone()
            rows = slice(1, 2) if name in ("final", "dh0") else slice(150, 450)
            got[rows, 5], got[rows, 9] = value[rows, 5], value[rows, 9]
            assert torch.equal(got, value), (name, bad)


def test_thousands_of_short_sequences(dgn):
    check(dgn, make([0, 1, 2] * 1500, 6, 1, "sigmoid", "bf16"), 6, 1, "sigmoid", "bf16", "thousands")
    check(dgn, make([1] * 30 + [0] * 4300 + [2, 0, 0], 70, 1, "decay", "f32"), 70, 1, "decay", "f32", "thousands empty")


@pytest.mark.parametrize("heads,group", [(2048, 1), (16, 128)])
def test_results_past_the_caches(dgn, heads, group):
    """Calls so large that their results are written past the caches, against each sequence alone (whose are not), on random
    rows.  Both round the same 32-bit values, cut in other places, to bf16: half a unit in the last place each, and the
    32-bit values differ by far less."""
    lens = [30000, 1, 0, 9999]
    n, c = sum(lens), heads * group
    torch.manual_seed(5)
    rn = lambda w: torch.randn(n, w, device="cuda").to(torch.bfloat16)  # noqa: E731
    x, gate, dy = rn(c), (rn(heads) * 1.5 + 2.0), rn(c)
    ptr = torch.tensor([0, 30000, 30001, 30001, n], device="cuda")
    b = dgn.ScanBuffers(n, 4, c, gate_group=group, kind="sigmoid", train=True)
    b.forward(x, gate, ptr)
    b.backward(x, gate, ptr, dy)
    for q, m in enumerate(lens):
        at, step = slice(int(ptr[q]), int(ptr[q]) + m), 64
        for head in (0, heads // 2):                     # a few heads of each sequence, so that the call is small
            few = max(1, step // group)
            h, ch = slice(head, head + few), slice(head * group, (head + few) * group)
            o = dgn.ScanBuffers(m, 1, few * group, gate_group=group, kind="sigmoid", train=True)
            one = torch.tensor([0, m], device="cuda")
            args = (x[at, ch], gate[at, h], one)
            o.forward(*args)
            o.backward(*args, dy[at, ch])
            for name, cols in (("y", ch), ("dx", ch), ("dgate", h)):
                got, want = getattr(b, name)[at, cols].float(), getattr(o, name).float()
                scale = want.abs().clamp(min=1e-2) if group == 1 else want.abs() + 1e-2 * group ** 0.5
                assert ((got - want).abs() <= 2.0 ** -7 * scale).all(), (name, q, head)
            torch.testing.assert_close(b.final[q, ch], o.final[0], rtol=1e-4, atol=1e-4)
            torch.testing.assert_close(b.dh0[q, ch], o.dh0[0], rtol=1e-4, atol=1e-4)


def test_long_sequences_and_repeats(dgn):
    """Longer than anything that one workgroup sees, twice: the same bits; many channels beside."""
    for kind, dtype, n, heads, group in [("sigmoid", "bf16", 9001, 6, 1), ("decay", "f32", 5000, 2, 130), ("decay", "f16", 7001, 3, 64)]:
        i = make([n, 500], heads, group, kind, dtype)
        b = check(dgn, i, heads, group, kind, dtype, "long")
        first = [t.clone() for t in (b.y, b.final, b.dx, b.dgate, b.dh0)]
        for _ in range(3):
            b.forward(i["x"], i["gate"], i["rowptr"], h0=i["h0"])
            b.backward(i["x"], i["gate"], i["rowptr"], i["dy"], h0=i["h0"], dfinal=i["dfinal"])
        assert all(torch.equal(s, t) for s, t in zip(first, (b.y, b.final, b.dx, b.dgate, b.dh0)))


def test_wide_batches_agree_with_each_sequence_alone(dgn):
    """Sizes at which the plain form would take too long: a packed batch against its sequences one at a time (which the
    other tests hold to the plain form), in 32 bits; the two may cut a sequence in other places."""
    lens = [1, 3000, 0, 777, 128, 2500]
    i = make(lens, 512, 1, "sigmoid", "f32")
    b = dgn.ScanBuffers(sum(lens), len(lens), 512, kind="sigmoid", dtype=torch.float32, train=True)
    b.forward(i["x"], i["gate"], i["rowptr"], h0=i["h0"])
    b.backward(i["x"], i["gate"], i["rowptr"], i["dy"], h0=i["h0"], dfinal=i["dfinal"])
    for q, n in enumerate(lens):
        at = slice(sum(lens[:q]), sum(lens[:q]) + n)
        o = dgn.ScanBuffers(n, 1, 512, kind="sigmoid", dtype=torch.float32, train=True)
        ptr, one = torch.tensor([0, n], device="cuda"), slice(q, q + 1)
        o.forward(i["x"][at], i["gate"][at], ptr, h0=i["h0"][one])
        o.backward(i["x"][at], i["gate"][at], ptr, i["dy"][at], h0=i["h0"][one], dfinal=i["dfinal"][one])
        for name in ("y", "dx", "dgate"):
            torch.testing.assert_close(getattr(b, name)[at], getattr(o, name), rtol=2e-5, atol=2e-5)
        for name in ("final", "dh0"):
            torch.testing.assert_close(getattr(b, name)[one], getattr(o, name), rtol=2e-5, atol=2e-5)


@pytest.mark.parametrize("kind", ["decay", "sigmoid"])
def test_gradients_against_differences(dgn, kind):
    """Central differences, in 64 bits, of the loss that dy and dfinal are the gradient of.  Room: what the gradients may be off
    by the bounds above (under 2e-5 of the sum of absolute products here), and the differences' own 1e-6."""
    group, i = 4, make([90, 0, 201], 9, 4, kind, "f32")
    b = check(dgn, i, 9, group, kind, "f32", "differences")
    gen = torch.Generator().manual_seed(9)
    for name, grad in [("x", b.dx), ("gate", b.dgate), ("h0", b.dh0)]:
        way = torch.randn(i[name].shape, generator=gen, dtype=torch.float64)

        def loss(step):
            moved = {k: i[k].double().cpu() + (step * way if k == name else 0.0) for k in ("x", "gate", "h0")}
            r = vo.scan(moved["x"], moved["gate"], i["rowptr"], kind, group, moved["h0"])
            return float((r["y"][0] * i["dy"].double().cpu()).sum() + (r["final"][0] * i["dfinal"].double().cpu()).sum())
        want, parts = (loss(1e-5) - loss(-1e-5)) / 2e-5, grad.double().cpu() * way
        assert abs(want - float(parts.sum())) <= (2e-5 + 1e-6) * float(parts.abs().sum()), name


@pytest.mark.parametrize("rows", [1, 3, 64, 200])
@pytest.mark.parametrize("heads,group", [(1, 1), (37, 1), (500, 1), (3, 64), (2, 33)])
def test_one_token(dgn, rows, heads, group):
    for kind, dtype in [("decay", "bf16"), ("sigmoid", "f16"), ("sigmoid", "f32"), ("decay", "f32")]:
        i = make([1] * rows, heads, group, kind, dtype)
        c, slots = heads * group, rows + 5
        gen = torch.Generator().manual_seed(rows)
        slot = torch.randperm(slots, generator=gen)[:rows].to(torch.int32)
        if rows > 2:
            slot[1], slot[-1] = -1, slots + 3           # idle, and outside the pool
        pool = torch.randn(slots, c, generator=gen)
        idle = (slot < 0) | (slot >= slots)
        i["h0"] = torch.where(idle[:, None], 0.0, pool[slot.clamp(0, slots - 1).long()]).cuda()
        want = vo.scan(i["x"], i["gate"], i["rowptr"], kind, group, i["h0"])
        for y_at in (None, "same"):
            b = dgn.ScanStepBuffers(rows, slots, c, gate_group=group, kind=kind, dtype=TYPES[dtype])
            state, out = pool.cuda(), torch.full((slots, c), 5.0, device="cuda")
            b.step(i["x"], i["gate"], slot.cuda(), state, out if y_at is None else None)
            after = out if y_at is None else state
            vo.within(b.y[~idle], want["y"][0][~idle], want["y"][1][~idle], "y")
            assert (b.y[idle] == 0).all()
            live = slot[~idle].long()
            vo.within(after[live.cuda()], want["final"][0][~idle], want["final"][1][~idle], "state")
            rest = torch.ones(slots, dtype=torch.bool)
            rest[live] = False
            keep = torch.full((slots, c), 5.0) if y_at is None else pool
            assert torch.equal(after.cpu()[rest], keep[rest]), "a state that no row has"


def test_one_token_of_every_row_in_turn(dgn):
    """Without slots row r has state r; token by token it gives what the scan gives."""
    i = make([40] * 6, 90, 1, "sigmoid", "f32")
    b, s = dgn.ScanBuffers(240, 6, 90, kind="sigmoid", dtype=torch.float32), dgn.ScanStepBuffers(6, 6, 90, dtype=torch.float32)
    b.forward(i["x"], i["gate"], i["rowptr"], h0=i["h0"])
    state = i["h0"].clone()
    x, g, y = (t.view(6, 40, 90) for t in (i["x"], i["gate"], b.y))
    for t in range(40):
        s.step(x[:, t], g[:, t], None, state)           # rows 40 * 90 elements apart
        torch.testing.assert_close(s.y, y[:, t], rtol=1e-5, atol=1e-5)
    torch.testing.assert_close(state, b.final, rtol=1e-5, atol=1e-5)


def test_offsets_past_32_bits(dgn):
    """Rows so far apart that the last ones lie more than 2^32 bytes behind the first."""
    rows, stride = 300, 2**24
    store = torch.empty((rows - 1) * stride + 64, dtype=torch.bfloat16, device="cuda")
    gate = store.as_strided((rows, 30), (stride, 1))
    small = make([rows], 30, 1, "sigmoid", "bf16")
    gate.copy_(small["gate"])
    small["gate"] = gate
    check(dgn, small, 30, 1, "sigmoid", "bf16", "far")


def test_another_stream_and_a_captured_graph(dgn):
    i = make([900, 0, 333], 100, 1, "sigmoid", "bf16")
    b = check(dgn, i, 100, 1, "sigmoid", "bf16", "stream")
    want = [t.clone() for t in (b.y, b.final, b.dx, b.dgate, b.dh0)]
    outs = lambda: (b.y, b.final, b.dx, b.dgate, b.dh0)  # noqa: E731

    def run(stream=None):
        b.forward(i["x"], i["gate"], i["rowptr"], h0=i["h0"], stream=stream)
        b.backward(i["x"], i["gate"], i["rowptr"], i["dy"], h0=i["h0"], dfinal=i["dfinal"], stream=stream)
    side = torch.cuda.Stream()
    for t in outs():
        t.zero_()
    torch.cuda.synchronize()
    run(side)
    side.synchronize()
    assert all(torch.equal(s, t) for s, t in zip(want, outs()))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for turn in range(4):
        for t in outs():
            t.fill_(float(turn))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(s, t) for s, t in zip(want, outs())), turn


def test_refusals_of_the_buffers(dgn):
    b = dgn.ScanBuffers(20, 2, 12, gate_group=3, kind="decay", train=True)
    i = make([12, 8], 4, 3, "decay", "bf16")
    good = dict(x=i["x"], gate=i["gate"], seq_rowptr=i["rowptr"], h0=i["h0"])
    b.forward(**good)
    for name, bad in [("x", i["x"].float()), ("x", i["x"][:, :11]), ("x", i["x"][:19]), ("x", i["x"].cpu()), ("gate", i["x"]),
                      ("x", i["x"].t().contiguous().t()), ("seq_rowptr", i["rowptr"].int()), ("seq_rowptr", i["rowptr"][:2]),
                      ("h0", i["h0"].half()), ("h0", i["h0"][:1]), ("x", i["x"][:1].expand(20, 12)), ("x", 64)]:
        with pytest.raises(dgn.DgnError):
            b.forward(**{**good, name: bad})
    with pytest.raises(dgn.DgnError):
        b.backward(i["x"], i["gate"], i["rowptr"], i["dy"].float())
    with pytest.raises(dgn.DgnError):
        dgn.ScanBuffers(20, 2, 12).backward(i["x"], i["x"], i["rowptr"], i["dy"])
    for kw in [dict(gate_group=5), dict(kind="other"), dict(dtype=torch.float64), dict(gate_group=0)]:
        with pytest.raises((dgn.DgnError, ZeroDivisionError)):
            dgn.ScanBuffers(20, 2, 12, **kw)
    s = dgn.ScanStepBuffers(20, 30, 12, gate_group=3, kind="decay")
    pool = torch.zeros(30, 12, device="cuda")
    for args in [(i["x"], i["gate"], None, pool[:29]), (i["x"], i["gate"], torch.zeros(20, device="cuda"), pool),
                 (i["x"], i["gate"], None, pool.half()), (i["x"].half(), i["gate"], None, pool)]:
        with pytest.raises(dgn.DgnError):
            s.step(*args)
