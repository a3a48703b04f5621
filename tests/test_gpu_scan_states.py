"""States of the gated linear recurrence that are handed on: where they come in and go out, and links of growing gates."""
import pytest
import torch

from test_gpu_scan import TYPES, check, dgn, make  # noqa: F401

pytestmark = pytest.mark.gpu
GOING_ON = [[40], [100], [129, 0, 1000, 5], [9000, 1, 0, 700]]      # one strip, one launch, two launches, three


def buffers(dgn, i, heads, group, kind, dtype, train=True):
    n, seqs = i["x"].shape[0], i["rowptr"].numel() - 1
    return dgn.ScanBuffers(n, seqs, heads * group, gate_group=group, kind=kind, dtype=TYPES[dtype], train=train)


@pytest.mark.parametrize("lens", GOING_ON)
@pytest.mark.parametrize("heads,group,kind,dtype", [(70, 1, "sigmoid", "bf16"), (3, 64, "decay", "f32")])
def test_states_go_out_where_they_come_in(dgn, lens, heads, group, kind, dtype):  # noqa: F811
    """h0 = final and dfinal = dh0 give the same bits as states that lie elsewhere."""
    i = make(lens, heads, group, kind, dtype)
    print(f"going on: {lens}, {heads} x {group}, {kind}, {dtype}", flush=True)
    a, b = (buffers(dgn, i, heads, group, kind, dtype) for _ in range(2))
    a.forward(i["x"], i["gate"], i["rowptr"], h0=i["h0"])
    b.final.copy_(i["h0"])
    b.forward(i["x"], i["gate"], i["rowptr"], h0=b.final)
    assert torch.equal(a.y, b.y) and torch.equal(a.final, b.final)
    a.backward(i["x"], i["gate"], i["rowptr"], i["dy"], h0=i["h0"], dfinal=i["dfinal"])
    b.dh0.copy_(i["dfinal"])
    b.backward(i["x"], i["gate"], i["rowptr"], i["dy"], h0=i["h0"], dfinal=b.dh0)
    for name in ("dx", "dgate", "dh0"):
        assert torch.equal(getattr(a, name), getattr(b, name)), name
    with pytest.raises(dgn.DgnError):
        b.backward(i["x"], i["gate"], i["rowptr"], i["dy"], h0=b.final)


def test_states_that_overlap_in_part(dgn):  # noqa: F811
    """Through the C entry: final a row of states further on than h0, and a row before it."""
    lens, c = [700, 3, 0, 290], 33
    i = make(lens, c, 1, "sigmoid", "f32")
    b = buffers(dgn, i, c, 1, "sigmoid", "f32", train=False)
    b.forward(i["x"], i["gate"], i["rowptr"], h0=i["h0"])
    for start, end in [(0, 1), (1, 0)]:
        store = torch.full((5, c), 9.0, device="cuda")
        before, after = store[start:start + 4], store[end:end + 4]
        before.copy_(i["h0"])
        y = torch.zeros_like(b.y)
        rc = dgn.dgn_scan_forward(b._d, i["x"], i["gate"], i["rowptr"], before, y, after, None, b._scratch, b._scratch_bytes)
        assert rc == 0 and torch.equal(after, b.final) and torch.equal(y, b.y), (start, end)


def test_a_captured_call_goes_on_at_every_replay(dgn):  # noqa: F811
    """A captured chunk whose state comes in where it goes out, replayed: the chunks of one long sequence."""
    chunk, turns, c = 300, 5, 64
    i = make([chunk * turns], c, 1, "sigmoid", "f32")
    whole, b = (dgn.ScanBuffers(n, 1, c, kind="sigmoid", dtype=torch.float32) for n in (chunk * turns, chunk))
    whole.forward(i["x"], i["gate"], i["rowptr"], h0=i["h0"])
    x, gate = torch.empty_like(i["x"][:chunk]), torch.empty_like(i["gate"][:chunk])
    ptr = torch.tensor([0, chunk], device="cuda")
    eager = dgn.ScanBuffers(chunk, 1, c, kind="sigmoid", dtype=torch.float32)
    x.copy_(i["x"][:chunk]), gate.copy_(i["gate"][:chunk])
    b.forward(x, gate, ptr, h0=b.final)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.forward(x, gate, ptr, h0=b.final)
    b.final.copy_(i["h0"])
    eager.final.copy_(i["h0"])
    for turn in range(turns):
        at = slice(turn * chunk, (turn + 1) * chunk)
        x.copy_(i["x"][at]), gate.copy_(i["gate"][at])
        torch.cuda.synchronize()
        graph.replay()
        eager.forward(x, gate, ptr, h0=eager.final.clone())
        torch.cuda.synchronize()
        assert torch.equal(b.y, eager.y) and torch.equal(b.final, eager.final), turn
        torch.testing.assert_close(b.y, whole.y[at], rtol=2e-5, atol=2e-5)
    torch.testing.assert_close(b.final, whole.final, rtol=2e-5, atol=2e-5)


@pytest.mark.parametrize("n,middle,at", [(10000, 5000, 960), (20001, 13000, 3200), (66001, 40000, 8704)])
def test_gates_whose_products_leave_the_range_of_floats(dgn, n, middle, at):  # noqa: F811
    """Products of up to 64 gates are in range, those of more are not, and states and gradients are, forward and backward, with
    sequences that begin in the middle; the last of the sizes has more than 1 024 strips of 64 rows."""
    i = make([middle, 0, n - middle], 8, 1, "decay", "f32")
    for name in ("x", "dy"):
        i[name][:middle, :7] = 0.0
    i["h0"][0, :7] = 0.0
    i["dfinal"][0, :7] = 0.0
    gate, tiny = i["gate"][:middle], 2.0 ** -60
    gate[:, :7] = 1.0
    gate[:, :2] = 0.5
    gate[at:at + 64, 0] = 2.0                   # states of 0 stay 0 ...
    gate[at:at + 160, 1] = 2.0                  # ... and here,
    gate[:1200, 4] = 1.1                        # and here
    for c, first in [(2, 2.0), (3, 2.0), (5, 0.5), (6, 0.5)]:
        gate[at:at + 140, c], gate[at + 140:at + 280, c] = first, 1.0 / first
    i["h0"][0, 2] = i["h0"][0, 3] = tiny         # states between 2^-60 and 2^80
    i["dfinal"][0, 5] = i["dfinal"][0, 6] = tiny
    gen = torch.Generator().manual_seed(1)
    i["x"][:middle, 3] = (torch.randn(middle, generator=gen) * 2.0 ** -70).cuda()
    i["dy"][:middle, 6] = (torch.randn(middle, generator=gen) * 2.0 ** -70).cuda()
    b = check(dgn, i, 8, 1, "decay", "f32", "products")
    for t in (b.y, b.dx, b.dgate):
        assert (t[:middle, [0, 1, 4]] == 0).all()
    assert float(b.y[:middle, 2].max()) == 2.0 ** 80 and float(b.final[0, 2]) == tiny
    assert float(b.dx[:middle, 5].max()) == 2.0 ** 80 and float(b.dh0[0, 5]) == tiny
