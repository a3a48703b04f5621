"""Dropout added to a residual, against the plain generator and, bit for bit where the draw decides, the plain sums."""
import pytest
import torch

import layer_oracle as lo
import values_oracle as vo

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def dgn():
    assert torch.cuda.is_available(), "these tests need the GPU"
    import paper_1707_08265_amd as d
    return d


def check(b, x, residual, dy, seed, step, rate, what):
    n = x.numel()
    key = torch.tensor([seed - 2**64 if seed >= 2**63 else seed, step - 2**64 if step >= 2**63 else step]).cuda()
    print(f"dropout {what}: {tuple(x.shape)} {x.dtype} rate {rate}", flush=True)
    b.forward(x, key, residual=residual)
    b.backward(dy, key)
    drop = int(rate * 65536 + 0.5)
    keep = torch.from_numpy(lo.draws(n, seed, step) >= drop).view(x.shape)
    scale = 65536 / (65536 - drop) if drop < 65536 else 0.0
    kept = torch.where(keep, x.double().cpu() * scale, 0.0)
    r = torch.zeros_like(kept) if residual is None else residual.double().cpu()
    vo.within(b.y, kept + r, 4 * vo.U32 * (kept.abs() + r.abs()), "y")
    grad = torch.where(keep, dy.double().cpu() * scale, 0.0)
    vo.within(b.dx, grad, 4 * vo.U32 * grad.abs(), "dx")
    assert (b.dx.cpu()[~keep] == 0).all()


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("rows,columns", [(1, 1), (1, 7), (1, 8), (3, 5), (9, 8), (2, 17), (70, 33), (16, 1000), (5, 2049)])
def test_sizes(dgn, rows, columns, dtype):
    gen = torch.Generator().manual_seed(columns)
    rn = lambda: torch.randn(rows, columns, generator=gen).to(TYPES[dtype]).cuda()  # noqa: E731
    for k, rate in enumerate((0.0, 0.1, 0.5, 1.0)):
        b = dgn.DropoutBuffers(rows, columns, rate, dtype=TYPES[dtype])
        for t in (b.y, b.dx):
            t.fill_(7.0)
        check(b, rn(), rn() if k % 2 else None, rn(), 2**64 - 1 - k, 2**40 + k if k < 3 else 2**64 - 1, rate, "sizes")


def test_rows_with_gaps_and_odd_addresses(dgn):
    for dtype in TYPES:
        for columns in (13, 16, 64):
            wide = torch.randn(31, 3 * columns + 11).to(TYPES[dtype]).cuda()
            x, r, dy = wide[:, 1:columns + 1], wide[:, columns + 2:2 * columns + 2], wide[:, 2 * columns + 5:3 * columns + 5]
            check(dgn.DropoutBuffers(31, columns, 0.3, dtype=TYPES[dtype]), x, r, dy, 5, 6, 0.3, "gaps")


def test_in_place_and_what_dropped_places_hold(dgn):
    key = torch.tensor([3, 4]).cuda()
    for dtype, t in TYPES.items():
        x, r = torch.randn(40, 50).to(t).cuda(), torch.randn(40, 50).to(t).cuda()
        b = dgn.DropoutBuffers(40, 50, 0.4, dtype=t)
        b.forward(x, key, residual=r)
        want = b.y.clone()
        keep = torch.from_numpy(lo.draws(2000, 3, 4) >= int(0.4 * 65536 + 0.5)).view(40, 50)
        x.masked_fill_(~keep.cuda(), float("nan"))
        b.forward(x, key, residual=r)
        assert torch.equal(b.y, want)
        d = dgn.dgn_dropout_desc(num_rows=40, num_columns=50, dtype=dgn.values.DTYPES[t], rate=0.4)
        for out in (x, r):
            x2, r2 = x.clone(), r.clone()
            to = x2 if out is x else r2
            assert dgn.dgn_dropout(d, x2, r2, key, to) == 0
            assert torch.equal(to, want)


def test_steps_and_seeds_differ_and_the_share_is_right(dgn):
    n, b = 1 << 20, dgn.DropoutBuffers(1024, 1024, 0.25, dtype=torch.float32)
    one, masks = torch.ones(1024, 1024, device="cuda"), []
    for key in ([1, 0], [1, 1], [2, 0], [2, 1]):
        b.forward(one, torch.tensor(key).cuda())
        masks.append(b.y != 0)
    for m in masks:             # (of n draws with p = 1/4: within six standard deviations)
        assert abs(int((~m).sum()) - n / 4) < 6 * (n * 3 / 16) ** 0.5
    for i in range(4):
        for j in range(i):      # (both drop, or neither does: 10 of 16)
            assert abs(int((masks[i] == masks[j]).sum()) - n * 10 / 16) < 6 * (n * 60 / 256) ** 0.5


def test_captured_steps_take_their_number_from_memory(dgn):
    x, r = torch.randn(100, 70).bfloat16().cuda(), torch.randn(100, 70).bfloat16().cuda()
    b, key = dgn.DropoutBuffers(100, 70, 0.2), torch.tensor([9, 0]).cuda()
    b.forward(x, key, residual=r)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.forward(x, key, residual=r)
        b.backward(x, key)
    seen = []
    for k in range(4):
        key[1] = k + 100
        b.forward(x, key, residual=r)
        b.backward(x, key)
        want = b.y.clone(), b.dx.clone()
        b.y.zero_(), b.dx.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(b.y, want[0]) and torch.equal(b.dx, want[1])
        seen.append(want[0])
    assert not torch.equal(seen[0], seen[1])


def test_more_elements_than_one_launch_counts_in_32_bits(dgn):
    """Elements past 2^32: the last blocks' numbers need the second word of the counter's first half only past 2^35, but their
    addresses are past 2^32."""
    rows, columns = (1 << 32) // 4096 + 3, 4096
    x = torch.ones(rows, columns, dtype=torch.bfloat16, device="cuda")
    b = dgn.DropoutBuffers(rows, columns, 0.5)
    b.forward(x, torch.tensor([7, 8]).cuda())
    first = (rows * columns - 8000) // 8
    want = []
    for block in range(first, first + 1000):
        want += [p for w in lo.philox((block & 0xFFFFFFFF, block >> 32, 8, 0), (7, 0)) for p in (w & 0xFFFF, w >> 16)]
    got = b.y.view(-1)[-8000:].cpu()
    assert torch.equal(got != 0, torch.tensor(want) >= 32768)
    b.forward(x, torch.tensor([7, 8]).cuda(), residual=x)
    assert torch.equal(b.y.view(-1)[-8000:].cpu(), torch.where(torch.tensor(want) >= 32768, 3.0, 1.0).bfloat16())
