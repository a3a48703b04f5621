"""Selective scan on the GPU against its plain form in 64 bits (bounds: layer_oracle)."""
import pytest
import torch

import layer_oracle as lo
import values_oracle as vo

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
NAN = float("nan")
ROWS = ("x", "delta", "B", "C", "z")
GRADS = ("dx", "ddelta", "dA", "dB", "dC", "dD", "ddelta_bias", "dz", "dh0")


@pytest.fixture(scope="module")
def dgn():
    assert torch.cuda.is_available(), "these tests need the GPU"
    import paper_1707_08265_amd as d
    return d


def make(lens, c, states, groups, dtype, seed=0, pad=(0, 0), h0=True, z=True, D=True, bias=True):
    """Inputs on the GPU, the gradients that come in, and the sizes; rows of no sequence hold NaN."""
    gen = torch.Generator().manual_seed(seed)
    n, s, t = sum(lens), len(lens), TYPES[dtype]
    rn = lambda *shape: torch.randn(*shape, generator=gen)  # noqa: E731

    def rows(v):
        full = torch.full((pad[0] + n + pad[1], v.shape[1]), NAN)
        full[pad[0]:pad[0] + n] = v
        return full.to(t).cuda()
    i = dict(x=rows(rn(n, c)), delta=rows(rn(n, c)), A=-torch.exp(rn(c, states) * 0.7).cuda(), B=rows(rn(n, groups * states)),
             C=rows(rn(n, groups * states)), D=rn(c).cuda() if D else None, delta_bias=(rn(c) * 0.5 - 2).cuda() if bias else None,
             z=rows(rn(n, c)) if z else None, h0=rn(s, c, states).cuda() if h0 else None,
             seq_rowptr=torch.tensor([pad[0]] + [pad[0] + sum(lens[:k + 1]) for k in range(s)]).cuda())
    return i, rows(rn(n, c)), rn(s, c, states).cuda() if h0 else None


def buffers(dgn, i, groups, train=True):
    n, c = i["x"].shape
    return dgn.SelectiveBuffers(n, i["seq_rowptr"].numel() - 1, c, num_states=i["A"].shape[1], num_groups=groups, dtype=i["x"].dtype,
                                train=train)


def oracle(i, groups, dy=None, dfinal=None):
    names = {"seq_rowptr": "rowptr"}
    return lo.select(**{names.get(k, k): v for k, v in i.items()}, groups=groups, dy=dy, dfinal=dfinal)


def check(dgn, made, groups, what, train=True):
    i, dy, dfinal = made
    b = buffers(dgn, i, groups, train)
    n, c = i["x"].shape
    print(f"select {what}: {n} rows of {c} x {i['A'].shape[1]} in {groups}, {b.num_seqs} sequences, {i['x'].dtype}", flush=True)
    names = ["y"] + (["dx", "ddelta", "dB", "dC", "dz"] if train else [])
    for name in names:
        getattr(b, name).fill_(7.0)
    b.forward(**i)
    if train:
        b.backward(**i, dy=dy, dfinal=dfinal)
    torch.cuda.synchronize()
    want = oracle(i, groups, dy if train else None, dfinal)
    first, last = int(i["seq_rowptr"][0]), int(i["seq_rowptr"][-1])
    for name, (value, error) in want.items():
        got = getattr(b, name)
        if name in names:
            assert (got[:first] == 7.0).all() and (got[last:] == 7.0).all(), f"{what}: {name} outside the sequences"
            got, value, error = got[first:last], value[first:last], error[first:last]
        vo.within(got, value, error, f"{what}: {name}")
    return b


LENGTHS = {"one": [1], "two": [2], "none": [0], "strip": [16], "past": [17], "short": [15], "mixed": [0, 31, 1, 0, 0, 32, 33, 0, 2],
           "ones": [1] * 70, "long": [333], "pair": [70, 0, 3, 117], "63": [3] * 63, "64": [2] * 64, "65": [1, 0, 4, 1, 2] * 13, "many": [5, 0, 16, 17, 1, 33] * 3, "wide": [64, 63, 65, 128]}


@pytest.mark.parametrize("lens", sorted(LENGTHS))
@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_lengths(dgn, dtype, lens):
    check(dgn, make(LENGTHS[lens], 21, 16, 1, dtype), 1, lens)
    check(dgn, make(LENGTHS[lens], 21, 5, 3, dtype, seed=1, z=False), 3, lens)


@pytest.mark.parametrize("c,groups", [(1, 1), (2, 2), (15, 1), (16, 1), (17, 1), (64, 1), (65, 5), (66, 2), (130, 2), (257, 1), (300, 3)])
def test_channels(dgn, c, groups):
    for dtype, states in [("bf16", 16), ("f32", 4)]:
        check(dgn, make([50, 0, 23], c, states, groups, dtype, seed=c), groups, "channels")


@pytest.mark.parametrize("states", [1, 2, 3, 4, 5, 8, 9, 15, 16, 17, 24, 31, 32, 33, 64, 65, 100, 128, 200, 256])
def test_states(dgn, states):
    for dtype, groups in [("bf16", 1), ("f32", 2)]:
        check(dgn, make([40, 0, 23], 6, states, groups, dtype, seed=states), groups, "states")


@pytest.mark.parametrize("h0", [False, True])
@pytest.mark.parametrize("train", [False, True])
def test_options_and_room_for_more_rows(dgn, h0, train):
    for k, pad in enumerate([(0, 0), (3, 100), (70, 1), (16, 16)]):
        check(dgn, make([5, 0, 90], 20, 16, 1, "bf16", pad=pad, h0=h0, z=k != 1, D=k != 2, bias=k != 3), 1, f"pad {pad}", train)
        check(dgn, make([5, 0, 90], 20, 16, 1, "f32", pad=pad, h0=h0, z=k == 0, D=k == 1, bias=k == 2), 1, f"pad {pad}", train)


@pytest.mark.parametrize("c,states,groups", [(130, 64, 1), (70, 128, 2), (41, 256, 1), (90, 32, 1), (100, 100, 2)])
def test_channels_of_several_workgroups(dgn, c, states, groups):
    """Sums over channels that more than one workgroup of the backward pass has, with many states."""
    for dtype in ("bf16", "f32"):
        check(dgn, make([33, 0, 20], c, states, groups, dtype, seed=c), groups, "several workgroups")


def test_rows_with_gaps_and_odd_addresses(dgn):
    for dtype in TYPES:
        i, dy, dfinal = make([80, 41], 34, 12, 1, dtype)
        wide = torch.full((121, 5 * 40 + 7), NAN, dtype=TYPES[dtype], device="cuda")
        for k, name in enumerate(ROWS):
            t = i[name]
            i[name] = wide[:, 40 * k + 1:40 * k + 1 + t.shape[1]]
            i[name].copy_(t)
        check(dgn, (i, dy, dfinal), 1, "gaps")


# rows, channels, states: strips that a launch between them puts together, few and many of them a wave; and enough waves that a lane has 16
# states, with one lane a channel and several
STRIPS = [(5000, 70, 16, "bf16"), (2200, 130, 8, "f32"), (1500, 33, 64, "f16"), (20000, 24, 16, "f32"), (1000, 1090, 16, "bf16"),
          (600, 2200, 12, "f32"), (4100, 1090, 16, "f16"), (950, 610, 32, "bf16"), (1100, 530, 20, "f32"), (700, 300, 64, "bf16"),
          (450, 310, 64, "f32"), (700, 150, 128, "f16"), (900, 131, 100, "f32"), (700, 80, 256, "bf16"), (500, 77, 201, "f32")]


def test_many_strips(dgn):
    """More strips than a workgroup of the launch between them has, sequences that span them, and a few channels in full."""
    for rows, c, states, dtype in STRIPS:
        lens = [rows // 3, 1, 0, rows - rows // 3 - 1]
        i, dy, dfinal = make(lens, c, states, 1, dtype, seed=rows)
        b = buffers(dgn, i, 1)
        print(f"select many strips: {rows} x {c} x {states} {dtype}", flush=True)
        b.forward(**i)
        b.backward(**i, dy=dy, dfinal=dfinal)
        at = torch.tensor([0, c // 2, c - 1]).cuda()
        small = {k: v if k in ("B", "C", "seq_rowptr") else v[at] if k in ("A", "D", "delta_bias") else v[:, at].contiguous() for k, v in i.items()}
        want = oracle(small, 1, dy[:, at], dfinal[:, at])
        for name, (value, error) in want.items():
            if name in ("dB", "dC"):
                continue                                        # (sums over all channels: test_channels)
            got = getattr(b, name)
            vo.within(got[at] if name in ("dA", "dD", "ddelta_bias") else got[:, at], value, error, name)


def test_steps_and_decays_at_their_limits(dgn):
    """Steps of nearly 0 and large ones, decays of 0 and of everything, outer gates that are closed or wide open."""
    for dtype in ("f32", "bf16"):
        i, dy, dfinal = make([200], 24, 16, 1, dtype)
        i["delta"][:, 3] = torch.tensor([-80.0, 80.0, 0.0, -20.0], device="cuda").repeat(50)
        i["delta"][50:60, 7] = -100.0
        i["z"][:, 5] = torch.tensor([-200.0, 200.0, 0.0, -30.0], device="cuda").repeat(50)
        i["A"][2], i["A"][9] = 0.0, -1e4
        check(dgn, (i, dy, dfinal), 1, "limits")
        i["delta"][50:60, 7] = -float("inf")                    # a step of 0: the state stays
        b = buffers(dgn, i, 1)
        b.forward(**i)
        b.backward(**i, dy=dy, dfinal=dfinal)
        assert all(getattr(b, n).isfinite().all() for n in ("y", "final") + GRADS)


def test_what_is_no_number_stays_in_its_sequence_and_channel(dgn):
    names = ("y", "final") + GRADS
    for bad in (NAN, float("inf")):
        i, dy, dfinal = make([50, 100, 0, 40], 20, 16, 1, "bf16")
        clean = buffers(dgn, i, 1)
        clean.forward(**i)
        clean.backward(**i, dy=dy, dfinal=dfinal)
        want = {n: getattr(clean, n).clone() for n in names}
        i["x"][50 + 30, 5] = bad
        dy[50 + 30, 9] = bad
        b = buffers(dgn, i, 1)
        b.forward(**i)
        b.backward(**i, dy=dy, dfinal=dfinal)
        assert not b.y[80:150, 5].isfinite().all() and not b.dx[50:81, 9].isfinite().all()
        for name, value in want.items():
            got = getattr(b, name).clone()
            if name in ("dB", "dC"):                            # (sums over channels)
                got[50:150] = value[50:150]
            elif name in ("final", "dh0"):
                got[1, 5], got[1, 9] = value[1, 5], value[1, 9]
            elif name in ("dA", "dD", "ddelta_bias"):
                got[5], got[9] = value[5], value[9]
            else:
                got[50:150, 5], got[50:150, 9] = value[50:150, 5], value[50:150, 9]
            assert torch.equal(got, value), (name, bad)


def test_sequences_that_go_on_from_call_to_call(dgn):
    """final as h0, in two calls, then token by token in the pool: near the call over all rows."""
    for dtype in TYPES:
        lens = [90, 2, 31, 0]
        i, _, _ = make(lens, 40, 16, 2, dtype)
        want = oracle(i, 2)
        parts, begin = buffers(dgn, i, 2, train=False), i["seq_rowptr"].tolist()
        parts.final.copy_(i["h0"])
        rows = [[] for _ in lens]
        for lo_, hi in [(0, 20), (20, 90)]:
            part, ptr, at = {**i, "h0": parts.final}, [0], 0
            for name in ROWS:
                part[name] = torch.zeros_like(i[name])
            for q in range(4):
                m = max(0, min(hi, lens[q]) - lo_)
                for name in ROWS:
                    part[name][at:at + m] = i[name][begin[q] + lo_:begin[q] + lo_ + m]
                at += m
                ptr.append(at)
            part["seq_rowptr"] = torch.tensor(ptr).cuda()
            parts.forward(**part)
            for q in range(4):
                rows[q].append(parts.y[ptr[q]:ptr[q + 1]].clone())
        vo.within(torch.cat([r for q in rows for r in q]), *want["y"], "y in two calls")
        vo.within(parts.final, *want["final"], "final in two calls")
        step, pool, out = dgn.SelectiveStepBuffers(3, 4, 40, num_states=16, num_groups=2, dtype=TYPES[dtype]), i["h0"].clone(), []
        for k in range(31):
            slots = torch.tensor([2, 0, 1 if k < 2 else -1], dtype=torch.int32).cuda()
            at = [92 + k, k, 90 + min(k, 1)]
            token = {name: i[name][at] for name in ROWS}
            step.step(**token, A=i["A"], D=i["D"], delta_bias=i["delta_bias"], slots=slots, state_in=pool)
            out.append(step.y.clone())
            assert k < 2 or (step.y[2] == 0).all()
        out, (value, error) = torch.stack(out), want["y"]
        vo.within(out[:, 0], value[92:123], error[92:123], "steps")
        vo.within(out[:, 1], value[:31], error[:31], "steps")
        vo.within(out[:2, 2], value[90:92], error[90:92], "steps")
        vo.within(pool[1:3], want["final"][0][1:3], want["final"][1][1:3], "pool")
        assert torch.equal(pool[3], i["h0"][3])


@pytest.mark.parametrize("states", [1, 3, 8, 16, 30, 64, 128, 256])
def test_one_token(dgn, states):
    for dtype, c, groups, rows, slots in [("bf16", 1, 1, 1, 1), ("f16", 38, 2, 5, 9), ("f32", 130, 1, 7, 7)]:
        i, _, _ = make([rows], c, states, groups, dtype, seed=states, h0=False)
        gen = torch.Generator().manual_seed(1)
        pool = torch.randn(slots, c, states, generator=gen).cuda()
        at = torch.randperm(slots, generator=gen)[:rows].to(torch.int32)
        if rows > 2:
            at[1], at[2] = -1, slots
        del i["seq_rowptr"], i["h0"]
        old, out = pool.clone(), pool.clone()
        b = dgn.SelectiveStepBuffers(rows, slots, c, num_states=states, num_groups=groups, dtype=TYPES[dtype])
        print(f"select step: {rows} rows of {c} x {states}, {dtype}", flush=True)
        b.step(**i, slots=at.cuda(), state_in=pool, state_out=out)
        assert torch.equal(pool, old)
        for r, s in enumerate(at.tolist()):
            if not 0 <= s < slots:
                assert (b.y[r] == 0).all()
                continue
            one = {k: v[r:r + 1] if k in ROWS else v for k, v in i.items()}
            want = lo.select(**one, rowptr=torch.tensor([0, 1]), groups=groups, h0=old[s:s + 1])
            vo.within(b.y[r:r + 1], *want["y"], "y")
            vo.within(out[s:s + 1], *want["final"], "state")
        idle = sorted(set(range(slots)) - set(at.tolist()))
        assert torch.equal(out[idle], old[idle])
        b.step(**i, slots=at.cuda(), state_in=pool)             # in place: the same
        assert torch.equal(pool, out)
        if rows == slots:
            b.step(**i, slots=None, state_in=old)               # row r is slot r
            assert old.isfinite().all()


def test_the_same_inputs_give_the_same_bits(dgn):
    i, dy, dfinal = make([500, 3, 0, 900], 150, 16, 2, "bf16")
    b, seen = buffers(dgn, i, 2), None
    for _ in range(3):
        b.forward(**i)
        b.backward(**i, dy=dy, dfinal=dfinal)
        now = [getattr(b, n).clone() for n in ("y", "final") + GRADS]
        assert seen is None or all(torch.equal(p, q) for p, q in zip(now, seen))
        seen = now
    only = buffers(dgn, i, 2, train=False)                      # without states kept: the same
    only.forward(**i)
    assert torch.equal(only.y, seen[0]) and torch.equal(only.final, seen[1])


def test_no_rows_and_no_sequences(dgn):
    for tokens, seqs in [(0, 3), (12, 0), (0, 0)]:
        b = dgn.SelectiveBuffers(tokens, seqs, 8, num_states=4, train=True)
        for n in ("final", "dA", "dD", "ddelta_bias", "dh0"):
            getattr(b, n).fill_(7.0)
        x, w = torch.ones(tokens, 8, dtype=torch.bfloat16, device="cuda"), torch.ones(tokens, 4, dtype=torch.bfloat16, device="cuda")
        A, one, h = -torch.ones(8, 4, device="cuda"), torch.ones(8, device="cuda"), torch.ones(seqs, 8, 4, device="cuda")
        i = dict(x=x, delta=x, A=A, B=w, C=w, D=one, delta_bias=one, z=x, h0=h, seq_rowptr=torch.zeros(seqs + 1, dtype=torch.int64, device="cuda"))
        b.forward(**i)
        b.backward(**i, dy=x, dfinal=h)
        assert (b.dA == 0).all() and (b.dD == 0).all() and (b.ddelta_bias == 0).all()
        assert torch.equal(b.final, h) and torch.equal(b.dh0, h) and (b.y == 0).all() and (b.dx == 0).all()


def test_captured_and_replayed(dgn):
    i, dy, dfinal = make([300, 0, 64], 60, 16, 1, "bf16")
    b, names = buffers(dgn, i, 1), ("y", "final") + GRADS

    def step():
        b.forward(**i)
        b.backward(**i, dy=dy, dfinal=dfinal)
    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(3):
        i["x"].copy_(torch.randn(364, 60).cuda())
        step()
        want = [getattr(b, n).clone() for n in names]
        for n in names:
            getattr(b, n).zero_()
        graph.replay()
        torch.cuda.synchronize()
        for n, w in zip(names, want):
            assert torch.equal(getattr(b, n), w), (k, n)
