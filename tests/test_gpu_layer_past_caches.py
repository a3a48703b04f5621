"""The operators of a selective recurrent layer in calls that are larger than the last-level cache, whose results go past it: every
element type, number of taps and of states."""
import pytest
import torch

import layer_oracle as lo
import values_oracle as vo

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
CACHE = 256 << 20                   # bytes of the last-level cache


@pytest.fixture(scope="module")
def dgn():
    assert torch.cuda.is_available(), "these tests need the GPU"
    import paper_1707_08265_amd as d
    return d


def normal(seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return lambda *s: torch.randn(*s, generator=gen, device="cuda")


@pytest.mark.parametrize("states", [4, 8, 16, 32, 64, 128, 256])
@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_one_token_of_the_scan(dgn, dtype, states):
    """All rows of some channels, and some rows of all channels, in full; rows of no slot; slots of no row."""
    t, c, rn = TYPES[dtype], 1030, normal(states)
    n = CACHE // (c * (8 * states + 6)) + 13
    i = dict(x=rn(n, c).to(t), delta=rn(n, c).to(t), A=-torch.exp(rn(c, states)), B=rn(n, states).to(t), C=rn(n, states).to(t), D=rn(c),
             delta_bias=rn(c) - 2, z=rn(n, c).to(t))
    pool = rn(n + 7, c, states)
    slots = torch.randperm(n + 7, device="cuda", generator=torch.Generator(device="cuda").manual_seed(n)).to(torch.int32)[:n]
    idle = torch.arange(n, device="cuda") % 50 == 5
    slots[idle] = -1
    b = dgn.SelectiveStepBuffers(n, n + 7, c, num_states=states, dtype=t)
    print(f"select step: {n} rows of {c} x {states}, {dtype}", flush=True)
    out = torch.full_like(pool, 7.0)
    b.step(**i, slots=slots, state_in=pool, state_out=out)
    at, live = slots.long(), ~idle
    assert (b.y[idle] == 0).all()
    unused = torch.ones(n + 7, dtype=torch.bool, device="cuda")
    unused[at[live]] = False
    assert (out[unused] == 7.0).all() and out.isfinite().all() and b.y.isfinite().all()

    def compare(rows, channels):
        one = {k: v[rows] if k in ("B", "C") else v[channels] if k in ("A", "D", "delta_bias") else v[rows][:, channels] for k, v in i.items()}
        want = lo.select(**one, rowptr=torch.arange(len(rows) + 1), h0=pool[at[rows]][:, channels])
        vo.within(b.y[rows][:, channels], *want["y"], "y")
        vo.within(out[at[rows]][:, channels], *want["final"], "state")
    compare(live.nonzero()[:, 0], torch.tensor([0, 17, c // 2, c - 1]).cuda())
    compare(live.nonzero()[:, 0][[0, 3, n // 2, -1]], torch.arange(c).cuda())
    b.step(**i, slots=slots, state_in=pool)                 # in place: the same
    assert torch.equal(pool[~unused], out[~unused])


@pytest.mark.parametrize("act", ["none", "silu"])
@pytest.mark.parametrize("taps", [2, 3, 4])
@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_convolution(dgn, dtype, taps, act):
    t, rn = TYPES[dtype], normal(taps)
    c = 1025 if dtype != "f32" else 515
    rows = CACHE // (2 * c * (4 if dtype == "f32" else 2)) + 37
    x, w, bias, dy, s0, df = rn(rows, c).to(t), rn(c, taps), rn(c), rn(rows, c).to(t), rn(4, taps - 1, c).to(t), rn(4, taps - 1, c).to(t)
    ptr = torch.tensor([0, rows // 3, rows // 3, rows // 3 + 2, rows]).cuda()
    b = dgn.ConvBuffers(rows, 4, c, taps=taps, activation=act, dtype=t, train=True)
    print(f"conv: {rows} x {c}, {taps} taps, {act}, {dtype}", flush=True)
    b.forward(x, w, ptr, bias=bias, state0=s0)
    b.backward(x, w, ptr, dy, bias=bias, state0=s0, dfinal=df)
    some = torch.tensor([0, 1, c // 2, c - 2, c - 1]).cuda()
    want = lo.conv(x[:, some], w[some], bias[some], ptr, act, s0[..., some], dy[:, some], df[..., some])
    for name, (value, error) in want.items():
        got = getattr(b, name)
        vo.within(got[some] if name in ("dweight", "dbias") else got[..., some], value, error, name)
    assert b.y.isfinite().all() and b.dx.isfinite().all()


@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_dropout(dgn, dtype):
    t, rn, columns = TYPES[dtype], normal(1), 1031
    rows = CACHE // (2 * columns * (4 if dtype == "f32" else 2)) + 9
    n, drop = rows * columns, int(0.3 * 65536 + 0.5)
    x, r, key = rn(rows, columns).to(t), rn(rows, columns).to(t), torch.tensor([3, 2**40 + 1]).cuda()
    b = dgn.DropoutBuffers(rows, columns, 0.3, dtype=t)
    print(f"dropout: {rows} x {columns}, {dtype}", flush=True)
    b.forward(x, key, residual=r)
    b.backward(x, key)
    for first in (0, n // 16 * 8, n // 8 * 8 - 4000):       # (blocks of eight draws)
        words = [lo.philox((k, 0, 1, 1 << 8), (3, 0)) for k in range(first // 8, min(first // 8 + 500, -(-n // 8)))]
        draws = torch.tensor([p for four in words for v in four for p in (v & 0xFFFF, v >> 16)])[:n - first]
        part = lambda v: v.view(-1)[first:first + len(draws)].double().cpu()  # noqa: E731
        kept = torch.where(draws >= drop, part(x) * (65536 / (65536 - drop)), 0.0)
        vo.within(b.y.view(-1)[first:first + len(draws)], kept + part(r), 4 * vo.U32 * (kept.abs() + part(r).abs()), "y")
        vo.within(b.dx.view(-1)[first:first + len(draws)], kept, 4 * vo.U32 * kept.abs(), "dx")
    share = float((b.dx == 0).sum()) / n                    # (of n draws: within six standard deviations; x itself is hardly ever 0)
    assert abs(share - drop / 65536) < 6 * (0.3 * 0.7 / n) ** 0.5 + 1e-3
