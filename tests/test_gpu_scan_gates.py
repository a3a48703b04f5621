"""Gates of the recurrence by themselves, in 32 bits."""
import pytest
import torch

from test_gpu_scan import dgn  # noqa: F401

pytestmark = pytest.mark.gpu
U32 = 2.0 ** -24


@pytest.mark.parametrize("channels", [1000, 1001])
def test_gates_of_32_bits_are_rounded_not_approximated(dgn, channels):  # noqa: F811
    """sigma(g) from a state of 1 and an input of 0, 1 - sigma(g) from a state of 0 and an input of 1, by the one-token form and as the
    first row of a sequence.  Bound: the exponential's unit in the last place (2 U), the sum's and the quotient's roundings (U each),
    and the product's (U) for the smaller of the two, which has the exponential's error twice in part: 6 U."""
    gen = torch.Generator().manual_seed(7)
    rows = 40
    gate = (torch.rand(rows, channels, generator=gen) * 160 - 80).cuda()
    gate[0] = torch.linspace(-1, 1, channels)
    one = torch.ones(rows, channels, device="cuda")
    step = dgn.ScanStepBuffers(rows, rows, channels, kind="sigmoid", dtype=torch.float32)
    scan = dgn.ScanBuffers(rows, rows, channels, kind="sigmoid", dtype=torch.float32)
    ptr = torch.arange(rows + 1, device="cuda")
    for state, x, sign in [(one, 0 * one, 1), (0 * one, one, -1)]:
        want = torch.sigmoid(sign * gate.double())
        step.step(x, gate, None, state.clone())
        scan.forward(x, gate, ptr, h0=state)
        for got in (step.y, scan.y):
            off = (got.double() - want).abs() / want
            assert float(off.max()) <= 6 * U32, (sign, float(off.max()) / U32, float(gate.flatten()[off.argmax()]))
