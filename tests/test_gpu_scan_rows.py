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
