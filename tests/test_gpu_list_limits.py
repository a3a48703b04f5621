"""Norms, clipping and update over lists at the limits of their arguments."""
import pytest
import torch

from test_gpu_lists import ADAM, dgn, tensors  # noqa: F401

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")


@pytest.mark.parametrize("norms,max_norm,eps,want", [
    ([0.0, 0.0], 0.0, 0.0, [1.0, 1.0]),              # gradients of 0, nothing allowed: they stay 0
    ([0.0, 2.0], 0.0, 0.0, [1.0, 0.0]),
    ([0.0, 2.0], 1.0, 0.0, [1.0, 0.5]),
    ([INF, 2.0], INF, 0.0, [0.0, 1.0]),              # an infinite limit scales nothing, but for a norm that is infinite
    ([INF, NAN], INF, 1e-6, [0.0, NAN]),
    ([INF, 1e30], 1.0, 1e-6, [0.0, 1e-30]),
    ([NAN, 0.0], 0.0, 0.0, [NAN, 1.0]),
])
def test_factors_at_their_limits(dgn, norms, max_norm, eps, want):  # noqa: F811
    """Clipping by given norms, and the update's own factors (its first moment from 0 is (1 - beta1) f g)."""
    f32 = [torch.float32]
    g = [t.fill_(1.0) for t in tensors([300, 5000], f32)]
    out, words = tensors([300, 5000], f32, seed=1), torch.tensor([1, 2], device="cuda")
    lst = dgn.TensorList(g)
    b = dgn.GradientBuffers(lst, 2)
    b.norms.copy_(torch.tensor(norms))
    b.clip(dgn.TensorList(out), max_norm, eps=eps, mask=words)
    p, m, v = ([t.zero_() for t in tensors([300, 5000], f32)] for _ in range(3))
    dgn.AdamBuffers(lst, *(dgn.TensorList(t) for t in (p, m, v))).step(**ADAM, norms=b.norms, max_norm=max_norm, clip_eps=eps, mask=words)
    for i, f in enumerate(want):
        near = dict(rtol=2.0 ** -20, atol=0.0, equal_nan=True)
        torch.testing.assert_close(out[i], torch.full_like(out[i], f), **near)
        torch.testing.assert_close(m[i], torch.full_like(m[i], f * (1 - ADAM["beta1"])), **near)


def test_gradients_of_zero_stay_zero_when_nothing_is_allowed(dgn):  # noqa: F811
    g = [torch.zeros(n, device="cuda", dtype=torch.bfloat16) for n in (7, 5000)]
    lst = dgn.TensorList(g)
    b = dgn.GradientBuffers(lst)
    b.norm()
    b.clip(lst, 0.0, eps=0.0)
    assert all((t == 0).all() for t in g)


def test_a_mask_of_no_words_reaches_nothing(dgn):  # noqa: F811
    """The mask of a graph without tensors: ids lie outside of it, so no set needs any entry; without ids it is too short."""
    f32 = [torch.float32]
    g, p, m, v = (tensors([300, 5000], f32, seed=k) for k in range(4))
    old = [t.clone() for ts in (g, p, m, v) for t in ts]
    lst = dgn.TensorList(g)
    empty, ids = torch.zeros(0, dtype=torch.int64, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    b = dgn.GradientBuffers(lst, 3)
    a = dgn.AdamBuffers(lst, *(dgn.TensorList(t) for t in (p, m, v)))
    b.norm(empty, ids)
    assert (b.norms == 0).all()
    b.norms.fill_(50.0)
    b.clip(lst, 1.0, mask=empty, ids=ids)
    a.step(**ADAM, mask=empty, ids=ids)
    assert all(torch.equal(t, o) for t, o in zip([t for ts in (g, p, m, v) for t in ts], old))
    for call in (lambda: b.norm(empty), lambda: b.clip(lst, 1.0, mask=empty), lambda: a.step(**ADAM, mask=empty)):
        with pytest.raises(dgn.DgnError):
            call()


def test_a_list_keeps_the_memory_whose_addresses_it_has(dgn):  # noqa: F811
    """A tensor is given other memory after the list was made: what the list points to is not handed out to anybody else."""
    size = 3 << 20
    t = torch.nn.Parameter(torch.ones(size, device="cuda"))
    was = t.data_ptr()
    lst = dgn.TensorList([t])
    t.data = torch.full((size,), 2.0, device="cuda")
    others = [torch.zeros(size, device="cuda") for _ in range(4)]
    assert was not in [o.data_ptr() for o in others] + [t.data_ptr()]
    b = dgn.GradientBuffers(lst)
    b.norm()
    assert abs(float(b.norms[0]) - size ** 0.5) <= 2.0 ** -23 * size ** 0.5       # the old memory's, as it says
