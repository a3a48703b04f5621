"""Lists of a few small tensors, whose norms are one launch, up to the sizes from which they are two, against their plain forms in 64 bits."""
import pytest
import torch

import values_oracle as vo
from test_gpu_lists import ADAM, TYPES, dgn, signed, tensors, words_of  # noqa: F401

pytestmark = pytest.mark.gpu
SMALL = {"one": [1], "four": [4096, 3, 64, 1], "odd": [1, 0, 3, 4095, 4096, 4097, 7], "wide": [8192, 8191, 8193, 1, 0, 5000],
         "sixteen": [700] * 16, "seventeen": [701] * 17, "chunks": [129, 64, 1, 2] * 16, "past chunks": [129, 64, 1, 2] * 16 + [5],
         "elements": [8192] * 15 + [8191, 1], "past elements": [8192] * 16 + [1], "many": [4095] * 33}


@pytest.mark.parametrize("name", sorted(SMALL))
@pytest.mark.parametrize("sets", [1, 5, 64])
def test_norms_clipping_and_update_of_small_lists(dgn, name, sets):  # noqa: F811
    sizes, f32 = SMALL[name], [torch.float32]
    print(f"small list: {name}, {sets} sets", flush=True)
    g, out = tensors(sizes), tensors(sizes, seed=5)
    words = words_of(len(g), sets) if sets > 1 and len(g) > 1 else torch.ones(len(g), dtype=torch.int64)
    lst = dgn.TensorList(g)
    b = dgn.GradientBuffers(lst, sets)
    b.norms.fill_(9.0)
    b.norm(words.cuda())
    want = vo.norms(g, signed(words), sets)
    # 64-bit sums: what is left is the square root's rounding to 32 bits
    assert ((b.norms.double().cpu() - want).abs() <= 2.0 ** -23 * want).all()
    first = b.norms.clone()
    b.norm(words.cuda())
    assert torch.equal(first, b.norms)
    f = vo.factors(b.norms, signed(words), 0.05, 1e-6)
    b.clip(dgn.TensorList(out), 0.05, mask=words.cuda())
    p, m, v = (tensors(sizes, f32, seed=k) for k in range(3))
    for t in v:
        t.square_()
    old = [[t.clone() for t in ts] for ts in (p, m, v)]
    dgn.AdamBuffers(lst, *(dgn.TensorList(t) for t in (p, m, v))).step(**ADAM, norms=b.norms, max_norm=0.05, mask=words.cuda())
    for i, t in enumerate(g):
        scaled = t.double().cpu() * f[i]
        vo.within(out[i], scaled, 4 * vo.U32 * scaled.abs(), f"tensor {i}")
        if int(words[i]) == 0:
            assert all(torch.equal(n[i], o[i]) for n, o in zip((p, m, v), old))
            continue
        for n, (value, error), what in zip((p, m, v), vo.adam(*(o[i] for o in old), scaled, **ADAM), "pmv"):
            vo.within(n[i], value, error, f"{what} of tensor {i}")


def test_small_lists_by_ids_and_with_what_does_not_count(dgn):  # noqa: F811
    """A NaN in a tensor that a set does not need, each set's own sum, and tensors that stand for others of the graph."""
    g = tensors([5, 4096, 77, 300], [torch.float32])
    g[2].fill_(float("nan"))
    mask, ids = torch.tensor([0, 4, 3, 1, 0]).cuda(), torch.tensor([2, 3, 1, 9], dtype=torch.int32).cuda()
    b = dgn.GradientBuffers(dgn.TensorList(g), 3)
    b.norm(mask, ids)
    want = vo.norms(g[:2], [3, 1], 2)
    assert ((b.norms[:2].double().cpu() - want).abs() <= 2.0 ** -23 * want).all() and b.norms[2].isnan()
