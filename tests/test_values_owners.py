"""What the owners of buffers hand to the library, without a GPU."""
from types import SimpleNamespace

import torch

import paper_1707_08265_amd as dgn
from paper_1707_08265_amd import values


def test_a_mask_of_no_words_is_still_a_mask():
    lst = type("Two", (SimpleNamespace,), {"__len__": lambda self: 2})(index=-1, _mem=torch.zeros(64, dtype=torch.uint8))
    r = dgn.dgn_reach()
    values._fill_reach(r, lst, 1, torch.zeros(0, dtype=torch.int64), torch.zeros(2, dtype=torch.int32))
    assert r.num_words == 0 and r.tensor_mask and r.tensor_ids
