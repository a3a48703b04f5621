"""Short causal convolution on the GPU against its plain form in 64 bits (bounds: layer_oracle)."""
import pytest
import torch

import layer_oracle as lo
import values_oracle as vo

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
NAN = float("nan")


@pytest.fixture(scope="module")
def dgn():
    assert torch.cuda.is_available(), "these tests need the GPU"
    import paper_1707_08265_amd as d
    return d


def make(lens, c, taps, dtype, seed=0, pad=(0, 0), states=True, bias=True):
    gen = torch.Generator().manual_seed(seed)
    n, s, t = sum(lens), len(lens), TYPES[dtype]
    rn = lambda *shape: torch.randn(*shape, generator=gen)  # noqa: E731

    def rows(v):
        full = torch.full((pad[0] + n + pad[1], c), NAN)
        full[pad[0]:pad[0] + n] = v
        return full.to(t).cuda()
    rowptr = torch.tensor([pad[0]] + [pad[0] + sum(lens[:i + 1]) for i in range(s)]).cuda()
    i = dict(x=rows(rn(n, c)), weight=rn(c, taps).cuda(), seq_rowptr=rowptr)
    more = dict(bias=rn(c).cuda() if bias else None, state0=rn(s, taps - 1, c).to(t).cuda() if states else None)
    return i, more, rows(rn(n, c)), rn(s, taps - 1, c).to(t).cuda() if states else None


def check(dgn, made, taps, act, dtype, what, train=True):
    i, more, dy, dfinal = made
    n, c = i["x"].shape
    seqs = i["seq_rowptr"].numel() - 1
    print(f"conv {what}: {n} rows of {c}, {seqs} sequences, {taps} taps, {act}, {dtype}", flush=True)
    b = dgn.ConvBuffers(n, seqs, c, taps=taps, activation=act, dtype=TYPES[dtype], train=train)
    names = ["y"] + (["dx"] if train else [])
    for name in names:
        getattr(b, name).fill_(7.0)
    b.forward(**i, **more)
    if train:
        b.backward(**i, **more, dy=dy, dfinal=dfinal)
    torch.cuda.synchronize()
    want = lo.conv(i["x"], i["weight"], more["bias"], i["seq_rowptr"], act, more["state0"], dy if train else None, dfinal)
    first, last = int(i["seq_rowptr"][0]), int(i["seq_rowptr"][-1])
    for name, (value, error) in want.items():
        got = getattr(b, name)
        if name in names:
            assert (got[:first] == 7.0).all() and (got[last:] == 7.0).all(), f"{what}: {name} outside the sequences"
            got, value, error = got[first:last], value[first:last], error[first:last]
        vo.within(got, value, error, f"{what}: {name}")
    return b


LENGTHS = {"one": [1], "none": [0], "two": [2], "three": [3], "four": [4], "batch": [8], "past": [9], "run": [56, 57, 55], "ones": [1] * 130,
           "mixed": [0, 3, 1, 0, 0, 2, 64, 0], "few": [2, 1, 3, 0, 2, 2, 1] * 9, "long": [1291], "63": [2] * 63, "64": [1, 3] * 32, "65": [2] * 65, "empties": [5] + [0] * 150 + [7]}


@pytest.mark.parametrize("lens", sorted(LENGTHS))
@pytest.mark.parametrize("taps", [2, 3, 4])
def test_lengths(dgn, taps, lens):
    for dtype, act in [("f32", "silu"), ("f16", "none"), ("bf16", "silu")]:
        check(dgn, make(LENGTHS[lens], 37, taps, dtype), taps, act, dtype, lens)


@pytest.mark.parametrize("channels", [1, 2, 3, 4, 5, 127, 128, 129, 255, 256, 257, 1000])
def test_channels(dgn, channels):
    for dtype in TYPES:
        check(dgn, make([70, 0, 33], channels, 4, dtype, seed=channels), 4, "silu", dtype, "channels")


@pytest.mark.parametrize("states,bias", [(False, False), (False, True), (True, False)])
@pytest.mark.parametrize("train", [False, True])
def test_states_bias_and_room_for_more_rows(dgn, states, bias, train):
    for pad in [(0, 0), (3, 200), (130, 1)]:
        check(dgn, make([5, 0, 260], 40, 4, "bf16", pad=pad, states=states, bias=bias), 4, "silu", "bf16", f"pad {pad}", train)


def test_many_rows_in_runs_of_every_length(dgn):
    """Enough rows that a run has more than eight of them, up to the longest, and results that go past the caches."""
    for rows, c, dtype in [(9000, 1030, "bf16"), (9000, 530, "f32"), (70001, 1025, "f16")]:
        gen = torch.Generator(device="cuda").manual_seed(1)
        t = TYPES[dtype]
        rn = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
        rowptr = torch.tensor([0, rows // 3, rows // 3 + 1, rows]).cuda()
        x, w, bias, dy, s0 = rn(rows, c).to(t), rn(c, 4), rn(c), rn(rows, c).to(t), rn(3, 3, c).to(t)
        b = dgn.ConvBuffers(rows, 3, c, dtype=t, train=True)
        print(f"conv runs: {rows} x {c} {dtype}", flush=True)
        b.forward(x, w, rowptr, bias=bias, state0=s0)
        b.backward(x, w, rowptr, dy, bias=bias, state0=s0, dfinal=s0)
        some = torch.tensor([0, 1, c // 2, c - 2, c - 1])         # a channel is by itself: a few of them in full
        pick = lambda v: v[..., some.cuda()]  # noqa: E731
        want = lo.conv(pick(x), w[some.cuda()], bias[some.cuda()], rowptr, "silu", pick(s0), pick(dy), pick(s0))
        for name, (value, error) in want.items():
            got = getattr(b, name)
            vo.within(got[some.cuda()] if name in ("dweight", "dbias") else pick(got), value, error, name)


def test_rows_with_gaps_and_odd_addresses(dgn):
    for dtype in TYPES:
        i, more, dy, dfinal = make([100, 41], 66, 4, dtype)
        wide = torch.full((141, 2 * 66 + 5), NAN, dtype=TYPES[dtype], device="cuda")
        wide[:, 3:69], wide[:, 70:136] = i["x"], dy
        i["x"] = wide[:, 3:69]
        check(dgn, (i, more, wide[:, 70:136], dfinal), 4, "silu", dtype, "gaps")


def test_what_is_no_number_stays_in_its_sequence_channel_and_rows(dgn):
    for bad in (NAN, float("inf")):
        i, more, dy, dfinal = make([50, 60, 0, 40], 65, 4, "bf16")
        clean = check(dgn, (i, more, dy, dfinal), 4, "silu", "bf16", "clean")
        want = {n: getattr(clean, n).clone() for n in ("y", "final", "dx", "dweight", "dbias", "dstate0")}
        i["x"][109, 5] = bad                  # the last row of the second sequence
        dy[50, 9] = bad                       # and the first
        b = check(dgn, (i, more, dy, dfinal), 4, "silu", "bf16", "bad") if bad != bad else None
        if b is None:
            b = dgn.ConvBuffers(150, 4, 65, dtype=torch.bfloat16, train=True)
            b.forward(**i, **more)
            b.backward(**i, **more, dy=dy, dfinal=dfinal)
        hit = {"y": [(109, 5)], "dx": [(r, 5) for r in range(106, 110)] + [(50, 9)], "final": [(1, 2, 5)],
               "dstate0": [(1, j, 9) for j in range(3)], "dweight": [(5, j) for j in range(4)] + [(9, j) for j in range(4)],
               "dbias": [(5,), (9,)]}
        for name, value in want.items():
            got = getattr(b, name).clone()
            for at in hit[name]:
                got[at] = value[at]
            assert torch.equal(got, value), (name, bad)
        assert not b.y[109, 5].isfinite() and not b.dx[50, 9].isfinite()


def test_large_and_small_activations(dgn):
    i, more, dy, dfinal = make([200], 64, 4, "f32")
    i["x"][:, :8] *= torch.tensor([1e30, 1e4, 100.0, 30.0, 1e-3, 1e-20, 0.0, -90.0], device="cuda")
    check(dgn, (i, more, dy, dfinal), 4, "silu", "f32", "limits")


def test_sequences_that_go_on_from_call_to_call(dgn):
    """final as state0, and the same rows in one call and in three: the same bits; then token by token."""
    for dtype in TYPES:
        t = TYPES[dtype]
        (i, more, _, _), lens = make([90, 2, 31, 0], 130, 4, dtype), [90, 2, 31, 0]
        whole = dgn.ConvBuffers(123, 4, 130, dtype=t)
        whole.forward(**i, **more)
        parts = dgn.ConvBuffers(123, 4, 130, dtype=t)
        parts.final.copy_(more["state0"])
        begin = i["seq_rowptr"].tolist()
        cuts = [[min(v, n) for n in lens] for v in (0, 1, 30, 90)]
        rows = [[] for _ in lens]
        for lo_, hi in zip(cuts[:-1], cuts[1:]):
            x = torch.zeros(123, 130, dtype=t, device="cuda")
            ptr, at = [0], 0
            for q in range(4):
                m = hi[q] - lo_[q]
                x[at:at + m] = i["x"][begin[q] + lo_[q]:begin[q] + hi[q]]
                at += m
                ptr.append(at)
            parts.forward(x, i["weight"], torch.tensor(ptr).cuda(), bias=more["bias"], state0=parts.final)
            for q in range(4):
                rows[q].append(parts.y[ptr[q]:ptr[q + 1]].clone())
        assert torch.equal(torch.cat([r for q in rows for r in q]), whole.y)
        assert torch.equal(parts.final, whole.final)
        step = dgn.ConvStepBuffers(3, 4, 130, dtype=t)
        pool, out = more["state0"].clone(), []
        for k in range(31):
            slots = torch.tensor([0, 1 if k < 2 else -1, 2], dtype=torch.int32).cuda()
            x = torch.stack([i["x"][k], i["x"][90 + min(k, 1)], i["x"][92 + k]])
            step.step(x, i["weight"], slots, pool, bias=more["bias"])
            out.append(step.y.clone())
            assert k < 2 or (step.y[1] == 0).all()
        out = torch.stack(out)
        # (another kernel, whose last product and its rounding to 16 bits may be one operation)
        value, error = lo.conv(i["x"], i["weight"], more["bias"], i["seq_rowptr"], "silu", more["state0"])["y"]
        for got, at in [(out[:, 0], slice(0, 31)), (out[:2, 1], slice(90, 92)), (out[:, 2], slice(92, 123))]:
            vo.within(got, value[at], error[at], "steps")
        assert torch.equal(pool[1:3], whole.final[1:3]) and torch.equal(pool[3], more["state0"][3])


@pytest.mark.parametrize("taps", [2, 3, 4])
def test_one_token(dgn, taps):
    for dtype, c, rows, slots in [("bf16", 1, 1, 1), ("f16", 37, 5, 9), ("f32", 130, 7, 7), ("bf16", 1024, 33, 40)]:
        gen = torch.Generator().manual_seed(c)
        t = TYPES[dtype]
        rn = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
        wide = torch.full((rows, c + 3), NAN, dtype=t, device="cuda")
        wide[:, 1:c + 1] = rn(rows, c).to(t).cuda()
        x, w, bias, pool = wide[:, 1:c + 1], rn(c, taps).cuda(), rn(c).cuda(), rn(slots, taps - 1, c).to(t).cuda()
        at = torch.randperm(slots, generator=gen)[:rows].to(torch.int32)
        if rows > 2:
            at[1], at[2] = -1, slots
        old, out = pool.clone(), pool.clone()
        b = dgn.ConvStepBuffers(rows, slots, c, taps=taps, dtype=t)
        print(f"conv step: {rows} rows of {c}, {slots} slots, {dtype}", flush=True)
        b.step(x, w, at.cuda(), pool, out, bias=bias)
        assert torch.equal(pool, old)
        for r, s in enumerate(at.tolist()):
            if not 0 <= s < slots:
                assert (b.y[r] == 0).all()
                continue
            want = lo.conv(x[r:r + 1], w, bias, torch.tensor([0, 1]), "silu", old[s:s + 1])
            vo.within(b.y[r:r + 1], *want["y"], "y")
            assert torch.equal(out[s].double().cpu(), want["final"][0][0])
        idle = sorted(set(range(slots)) - set(at.tolist()))
        assert torch.equal(out[idle], old[idle])
        b.step(x, w, at.cuda(), pool, bias=bias)            # in place: the same
        assert torch.equal(pool, out)


def test_the_same_inputs_give_the_same_bits(dgn):
    made = make([700, 3, 0, 1500], 300, 4, "bf16")
    i, more, dy, dfinal = made
    b = dgn.ConvBuffers(2203, 4, 300, train=True)
    seen = None
    for _ in range(3):
        b.forward(**i, **more)
        b.backward(**i, **more, dy=dy, dfinal=dfinal)
        now = [getattr(b, n).clone() for n in ("y", "final", "dx", "dweight", "dbias", "dstate0")]
        assert seen is None or all(torch.equal(p, q) for p, q in zip(now, seen))
        seen = now


def test_no_rows_and_no_sequences(dgn):
    for tokens, seqs in [(0, 3), (12, 0), (0, 0)]:
        b = dgn.ConvBuffers(tokens, seqs, 8, train=True)
        for n in ("final", "dweight", "dbias", "dstate0"):
            getattr(b, n).fill_(7.0)
        x, s = torch.ones(tokens, 8, dtype=torch.bfloat16, device="cuda"), torch.ones(seqs, 3, 8, dtype=torch.bfloat16, device="cuda")
        w, ptr = torch.ones(8, 4, device="cuda"), torch.zeros(seqs + 1, dtype=torch.int64, device="cuda")
        b.forward(x, w, ptr, state0=s)
        b.backward(x, w, ptr, x, state0=s, dfinal=s)
        assert (b.dweight == 0).all() and (b.dbias == 0).all() and torch.equal(b.final, s) and torch.equal(b.dstate0, s)
        assert (b.y == 0).all() and (b.dx == 0).all()


def test_captured_and_replayed(dgn):
    i, more, dy, dfinal = make([300, 0, 64], 200, 4, "bf16")
    b = dgn.ConvBuffers(364, 3, 200, train=True)

    def step():
        b.forward(**i, **more)
        b.backward(**i, **more, dy=dy, dfinal=dfinal)
    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(3):
        i["x"].copy_(torch.randn(364, 200).cuda())
        step()
        want = [getattr(b, n).clone() for n in ("y", "final", "dx", "dweight", "dbias", "dstate0")]
        for n in ("y", "final", "dx", "dweight", "dbias", "dstate0"):
            getattr(b, n).zero_()
        graph.replay()
        torch.cuda.synchronize()
        for n, w in zip(("y", "final", "dx", "dweight", "dbias", "dstate0"), want):
            assert torch.equal(getattr(b, n), w), (k, n)
