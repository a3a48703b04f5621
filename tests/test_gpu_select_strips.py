"""Selective scan in strips of more than sixteen rows, as large calls have them, against its plain form in 64 bits: whole groups
of channels, with the gradients that are sums over them."""
import pytest
import torch

import layer_oracle as lo
import values_oracle as vo

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
NAN = float("nan")
ROWS, GROUPED = ("x", "delta", "z", "dy"), ("B", "C")
GRADS = ("dx", "ddelta", "dA", "dB", "dC", "dD", "ddelta_bias", "dz", "dh0")


@pytest.fixture(scope="module")
def dgn():
    assert torch.cuda.is_available(), "these tests need the GPU"
    import paper_1707_08265_amd as d
    return d


def strip_rows(dgn, tokens, c, states, groups, dtype):
    """Rows of a strip, from what a call asks for: with so many sequences, two states a strip, its sums, and a copy of h0."""
    seqs = 2**31 - 2
    d = dgn.dgn_select_desc(num_tokens=tokens, num_seqs=seqs, num_channels=c, num_states=states, num_groups=groups,
                            dtype=dgn.values.DTYPES[dtype])
    rc, need, _ = dgn.dgn_select_workspace(d)
    assert rc == 0
    wide = 4
    while wide < states:
        wide *= 2
    room = lambda v: -(-v // 256) * 256  # noqa: E731
    for rows in range(16, 80, 16):
        strips = -(-tokens // rows)
        if room(2 * room(strips * c * wide * 4) + room(strips * c * 4) + seqs * c * states * 4) == need:
            return rows
    raise AssertionError("strips of no known length")


# rows, groups, channels of a group, states, type, and the rows of a strip that this is to have: one or more lanes a channel, with four
# states each or 16; groups of one channel, of some, and of more than a wave or workgroup has
CASES = [(613, 512, 1, 16, "bf16", 64), (601, 450, 3, 4, "f32", 64), (500, 300, 2, 8, "f16", 32), (805, 256, 1, 12, "bf16", 48),
         (530, 512, 1, 32, "f32", 64), (530, 512, 1, 64, "f16", 64), (900, 300, 1, 128, "bf16", 64), (700, 300, 1, 256, "f32", 48),
         (500, 150, 70, 16, "bf16", 32), (600, 256, 40, 20, "f32", 64), (565, 160, 33, 64, "bf16", 64), (610, 450, 2, 5, "bf16", 64),
         (700, 300, 1, 3, "f16", 48)]


def check_long_strips(dgn, tokens, groups, share, states, dtype, rows):
    """Sequences that begin and end in any sixteen rows of a strip, some past several strips; rows of none before and after; the
    last strip is shorter."""
    t, c = TYPES[dtype], groups * share
    assert strip_rows(dgn, tokens, c, states, groups, t) == rows and tokens % 16
    before, after, lens = 21, 83, [40, 0, 17, 1, 33, 70, 0, 15, 16]
    lens.append(tokens - before - after - sum(lens))
    s, ptr = len(lens), torch.tensor([before] + [before + sum(lens[:k + 1]) for k in range(len(lens))]).cuda()
    gen = torch.Generator(device="cuda").manual_seed(tokens)
    rn = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")  # noqa: E731

    def full(width):
        v = rn(tokens, width)
        v[:before], v[tokens - after:] = NAN, NAN
        return v.to(t)
    i = dict(x=full(c), delta=full(c), A=-torch.exp(rn(c, states) * 0.7), B=full(groups * states), C=full(groups * states), D=rn(c),
             delta_bias=rn(c) * 0.5 - 2, z=full(c), h0=rn(s, c, states))
    dy, dfinal = full(c), rn(s, c, states)
    print(f"select strips of {rows}: {tokens} rows of {groups} x {share} x {states} {dtype}", flush=True)
    b = dgn.SelectiveBuffers(tokens, s, c, num_states=states, num_groups=groups, dtype=t, train=True)
    names = ("y", "dx", "ddelta", "dB", "dC", "dz")
    for name in names:
        getattr(b, name).fill_(7.0)
    b.forward(**i, seq_rowptr=ptr)
    b.backward(**i, seq_rowptr=ptr, dy=dy, dfinal=dfinal)
    torch.cuda.synchronize()
    inside = slice(before, tokens - after)
    for name in ("y", "final") + GRADS:
        got = getattr(b, name)
        if name in names:
            assert (got[:before] == 7.0).all() and (got[tokens - after:] == 7.0).all(), f"{name} outside the sequences"
            got = got[inside]
        assert got.isfinite().all(), name
    # some groups in full
    some = [0, groups // 2, groups - 1]
    at = torch.tensor([g * share + k for g in some for k in range(share)]).cuda()
    columns = torch.tensor([g * states + n for g in some for n in range(states)]).cuda()

    def pick(name, v):
        if name in ("B", "C", "dB", "dC"):
            return v[:, columns]
        return v[at] if name in ("A", "D", "delta_bias", "dA", "dD", "ddelta_bias") else v[:, at]
    want = lo.select(**{k: pick(k, v) for k, v in i.items()}, rowptr=ptr, groups=3, dy=pick("dy", dy), dfinal=pick("dfinal", dfinal))
    for name, (value, error) in want.items():
        got = pick(name, getattr(b, name))
        if name in names:
            got, value, error = got[inside], value[inside], error[inside]
        vo.within(got, value, error, name)
    only = dgn.SelectiveBuffers(tokens, s, c, num_states=states, num_groups=groups, dtype=t)       # without states kept: the same
    only.forward(**i, seq_rowptr=ptr)
    assert torch.equal(only.y[inside], b.y[inside]) and torch.equal(only.final, b.final)


@pytest.mark.parametrize("tokens,groups,share,states,dtype,rows", CASES)
def test_long_strips(dgn, tokens, groups, share, states, dtype, rows):
    check_long_strips(dgn, tokens, groups, share, states, dtype, rows)


@pytest.mark.parametrize("tokens,groups,share,states,dtype", [(1111, 256, 8, 256, "bf16"), (2201, 256, 5, 200, "f32"), (4100, 300, 1, 32, "f16"),
                                                              (1610, 300, 17, 128, "f32")])
def test_sums_over_channels_in_several_launches(dgn, tokens, groups, share, states, dtype):
    """Gradients whose sums over the channels of a group do not fit the scratch at once, with sequences that go on from launch to launch."""
    c, wide = groups * share, 32 if states <= 32 else 128 if states <= 128 else 256
    need = lambda only: dgn.dgn_select_workspace(dgn.dgn_select_desc(  # noqa: E731
        num_tokens=tokens, num_seqs=0, num_channels=c, num_states=states, num_groups=groups, dtype=dgn.values.DTYPES[TYPES[dtype]],
        forward_only=only))[1]
    blocks = groups * -(-share // (1024 // wide))
    strips = -(-tokens // 64)
    sums = need(0) - need(1) - strips * (c * wide + 2 * c) * 4
    assert sums < blocks * tokens * 2 * wide * 4 * 0.95
    check_long_strips(dgn, tokens, groups, share, states, dtype, 64)


@pytest.mark.parametrize("rows,c,states,dtype", [(100, 20, 9, "f32"), (100, 20, 16, "bf16"), (1300, 24, 5, "f32"), (2000, 40, 16, "f32"),
                                                 (1000, 1090, 12, "bf16")])
def test_steps_whose_sum_passes_the_range_of_floats(dgn, rows, c, states, dtype):
    """Two steps of 3e38 in a strip: what decays is gone, a state with an A of 0 stays, and numbers of states that are no power of two
    are as the others.  Few strips, and many that a launch between them puts together."""
    t, rn = TYPES[dtype], lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    gen = torch.Generator(device="cuda").manual_seed(rows)
    i = dict(x=rn(rows, c).to(t), delta=rn(rows, c).to(t), A=-torch.exp(rn(c, states) * 0.7), B=rn(rows, states).to(t),
             C=rn(rows, states).to(t), D=rn(c), delta_bias=rn(c) * 0.5 - 2, z=rn(rows, c).to(t), h0=rn(2, c, states))
    dy, dfinal = rn(rows, c).to(t), rn(2, c, states)
    i["A"][3] = 0.0
    for k in (35, 36, rows - 20, rows - 19):
        i["delta"][k, :8], i["x"][k, :8], i["B"][k] = 3e38, 0.0, 0.0
    ptr = torch.tensor([0, rows - 15, rows]).cuda()
    b = dgn.SelectiveBuffers(rows, 2, c, num_states=states, dtype=t, train=True)
    print(f"select long sums of steps: {rows} x {c} x {states} {dtype}", flush=True)
    b.forward(**i, seq_rowptr=ptr)
    b.backward(**i, seq_rowptr=ptr, dy=dy, dfinal=dfinal)
    at = torch.tensor([0, 3, 7, 8, c - 1]).cuda()
    pick = lambda n, v: v if n in ("B", "C") else v[at] if n in ("A", "D", "delta_bias", "dA", "dD", "ddelta_bias") else v[:, at]  # noqa: E731
    want = lo.select(**{k: pick(k, v) for k, v in i.items()}, rowptr=ptr, dy=dy[:, at], dfinal=dfinal[:, at])
    for name, (value, error) in want.items():
        if name in ("dB", "dC"):
            assert getattr(b, name).isfinite().all()
            continue
        got = pick(name, getattr(b, name))
        if name == "dA":                    # (of an A of 0: the sum of those steps times what is there, past the range too)
            keep = torch.tensor([0, 2, 3, 4])
            got, value, error = got[keep.cuda()], value[keep], error[keep]
        vo.within(got, value, error, name)


@pytest.mark.parametrize("rows,c,states,seqs", [(1, 20, 16, 3), (100, 33, 64, 5), (600, 300, 128, 9), (3000, 40, 256, 40), (2000, 1090, 5, 2)])
def test_the_forward_pass_stays_in_the_scratch_that_it_asks_for(dgn, rows, c, states, seqs):
    """With states that go out where they come in, whose copy is the last thing in it."""
    gen = torch.Generator(device="cuda").manual_seed(rows)
    rn = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    x, delta, B, C = rn(rows, c), rn(rows, c), rn(rows, states), rn(rows, states)
    A, h0 = -torch.exp(rn(c, states)), rn(seqs, c, states)
    ptr = torch.linspace(0, rows, seqs + 1).long().cuda()
    outs = []
    for only in (0, 1):
        m = dgn.dgn_select_desc(num_tokens=rows, num_seqs=seqs, num_channels=c, num_states=states, num_groups=1, dtype=dgn.DGN_F32,
                                forward_only=only)
        rc, need, _ = dgn.dgn_select_workspace(m)
        room, y, final = torch.full((need + 8192,), 7, dtype=torch.uint8, device="cuda"), torch.empty_like(x), h0.clone()
        scratch = room[4096:4096 + need]
        inputs = dgn.dgn_select_inputs(*(v if v is None else v.data_ptr() for v in (x, delta, A, B, C, None, None, None, ptr, final)))
        assert rc == 0 and dgn.dgn_select_forward(m, inputs, y, final, None, scratch, need) == 0
        assert (room[:4096] == 7).all() and (room[4096 + need:] == 7).all()
        outs += [(y, final)]
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])
    want = lo.select(x, delta, A, B, C, ptr, h0=h0) if rows * c * states < 4_000_000 else None
    if want:
        vo.within(outs[1][0], *want["y"], "y")
        vo.within(outs[1][1], *want["final"], "final")


@pytest.mark.parametrize("rows,c,states,groups", [(1, 20, 16, 1), (100, 33, 64, 3), (600, 300, 128, 1), (3000, 40, 256, 2), (700, 1090, 5, 1),
                                                  (2201, 1280, 200, 256)])
def test_the_gradients_stay_in_the_scratch_that_they_ask_for(dgn, rows, c, states, groups):
    """And what it holds before does not matter."""
    gen = torch.Generator(device="cuda").manual_seed(rows)
    rn = lambda *s: torch.randn(*s, generator=gen, device="cuda").bfloat16()  # noqa: E731
    i = dict(x=rn(rows, c), delta=rn(rows, c), A=-torch.exp(rn(c, states).float()), B=rn(rows, groups * states), C=rn(rows, groups * states))
    ptr, dy = torch.tensor([0, rows // 3, rows // 3, rows]).cuda(), rn(rows, c)
    b, seen = dgn.SelectiveBuffers(rows, 3, c, num_states=states, num_groups=groups, train=True), []
    for fill in (0, 255):                           # (of bytes of 255, floats are no numbers)
        room = torch.full((b._scratch_bytes + 8192,), fill, dtype=torch.uint8, device="cuda")
        b._scratch = room[4096:4096 + b._scratch_bytes]
        b.forward(**i, seq_rowptr=ptr)
        b._scratch.fill_(fill)
        b.backward(**i, seq_rowptr=ptr, dy=dy)
        assert (room[:4096] == fill).all() and (room[-4096:] == fill).all()
        seen.append([getattr(b, n).clone() for n in GRADS if n != "dz"])
    for name, one, two in zip([n for n in GRADS if n != "dz"], *seen):
        assert torch.equal(one, two) and one.isfinite().all(), name
