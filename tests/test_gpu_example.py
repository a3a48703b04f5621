"""The example: a training step from its pruned graph, the updater by target sets, and one token at a time."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_recurrent_training_from_the_pruned_graph():
    assert torch.cuda.is_available(), "these tests need the GPU"
    spec = importlib.util.spec_from_file_location("recurrent_training", os.path.join(ROOT, "examples", "recurrent_training.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    r = example.run(steps=60, head_steps=10)
    assert all(x == x for x in r.losses) and r.losses[59] < 0.3 * r.losses[0] and r.losses[-1] <= 1.1 * r.losses[59]
    # the second function has no gradient of the inner layer: its operators are gone and its parameters stay
    assert len(r.functions[0]) == 10 and len(r.functions[1]) == 6
    mask = r.mask.tolist()
    assert [mask[r.names[n]] for n in ("dw_in", "dw_gate", "dw_out")] == [1, 1, 3]
    assert torch.equal(r.before["w_in"], r.after["w_in"]) and torch.equal(r.before["w_gate"], r.after["w_gate"])
    assert not torch.equal(r.before["w_out"], r.after["w_out"])
    # served rows moved their states on, the others are as they were, the idle row answers zero
    moved = {4, 0, 3}
    for q in range(len(example.LENGTHS)):
        assert torch.equal(r.pool[q], r.final[q]) == (q not in moved), q
    assert (r.answer[2] == 0).all() and r.answer.isfinite().all() and (r.answer[[0, 1, 3]] != 0).any()
