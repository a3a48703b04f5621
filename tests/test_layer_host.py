"""Host-side checks of the operators of a selective recurrent layer that need no GPU: what the library refuses before any device
work, and the plain forms that the kernels are compared with."""
import ctypes

import numpy as np
import pytest
import torch

import layer_oracle as lo


@pytest.fixture(scope="module")
def d():
    import paper_1707_08265_amd as d
    return d


def conv_desc(d, **kw):
    base = dict(num_tokens=10, num_seqs=2, num_channels=12, num_taps=4, activation=d.DGN_ACT_SILU, dtype=d.DGN_BF16)
    return d.dgn_conv_desc(**{**base, **kw})


def select_desc(d, **kw):
    base = dict(num_tokens=10, num_seqs=2, num_channels=12, num_states=5, num_groups=3, dtype=d.DGN_BF16)
    return d.dgn_select_desc(**{**base, **kw})


def apart(names, start=1 << 20, step=1 << 20):
    """An address for each name, far enough from each other."""
    return {n: start + k * step for k, n in enumerate(names)}


def test_structures_have_the_sizes_of_the_header(d):
    assert ctypes.sizeof(d.dgn_conv_desc) == 3 * 8 + 4 * 4 + 4 * 8
    assert ctypes.sizeof(d.dgn_select_desc) == 5 * 8 + 2 * 4 + 12 * 8
    assert ctypes.sizeof(d.dgn_select_inputs) == 80 and ctypes.sizeof(d.dgn_select_grads) == 72
    assert ctypes.sizeof(d.dgn_dropout_desc) == 2 * 8 + 2 * 4 + 8 + 3 * 8


def test_conv_description_is_checked(d):
    rc, nb = d.dgn_conv_workspace(conv_desc(d))
    assert rc == 0 and nb > 0 and d.dgn_conv_workspace(None)[0] == d.DGN_ERR_NULL_PTR
    for bad, code in [(dict(num_tokens=-1), -1), (dict(num_seqs=-1), -1), (dict(num_channels=-1), -1), (dict(num_taps=1), -1),
                      (dict(num_taps=5), -1), (dict(activation=2), -1), (dict(dtype=3), -1), (dict(x_stride=11), -1),
                      (dict(dx_stride=-12), -1), (dict(num_tokens=2**31 - 1), -3), (dict(num_seqs=2**31), -3),
                      (dict(num_channels=2**31), -3), (dict(num_channels=2**29), -3), (dict(y_stride=2**41), -3)]:
        assert d.dgn_conv_workspace(conv_desc(d, **bad))[0] == code, bad
        if bad != dict(num_channels=2**29):
            assert d.dgn_conv_step(conv_desc(d, **bad), 4, 64, 64, None, None, 64, 64, 64, stream=0) == code, bad


def test_conv_calls_refuse_bad_pointers(d):
    m = conv_desc(d)
    nb = d.dgn_conv_workspace(m)[1]
    good = apart(("x", "weight", "bias", "seq_rowptr", "state0", "y", "final", "scratch"))
    forward = lambda scratch_bytes=nb, **kw: d.dgn_conv_forward(m, **{**good, **kw}, scratch_bytes=scratch_bytes, stream=0)  # noqa: E731
    for n in ("x", "weight", "seq_rowptr", "y", "scratch"):
        assert forward(**{n: None}) == d.DGN_ERR_NULL_PTR, n
    for n, off in [("x", 1), ("y", 1), ("weight", 2), ("bias", 2), ("seq_rowptr", 4), ("state0", 1), ("final", 1), ("scratch", 4)]:
        assert forward(**{n: good[n] + off}) == d.DGN_ERR_INVALID_ARG, n
    assert forward(nb - 1) == d.DGN_ERR_WORKSPACE_TOO_SMALL
    for out in ("y", "final", "scratch"):
        for n in good:
            if n != out and (out, n) != ("final", "state0"):
                assert forward(**{out: good[n]}) == d.DGN_ERR_INVALID_ARG, (out, n)
    good = apart(("x", "weight", "bias", "seq_rowptr", "state0", "dy", "dfinal", "dx", "dweight", "dbias", "dstate0", "scratch"))
    back = lambda scratch_bytes=nb, **kw: d.dgn_conv_backward(m, **{**good, **kw}, scratch_bytes=scratch_bytes, stream=0)  # noqa: E731
    for n in ("x", "weight", "seq_rowptr", "dy", "dx", "dweight", "scratch"):
        assert back(**{n: None}) == d.DGN_ERR_NULL_PTR, n
    for n, off in [("dy", 1), ("dx", 1), ("dfinal", 1), ("dstate0", 1), ("dweight", 2), ("dbias", 2), ("scratch", 4)]:
        assert back(**{n: good[n] + off}) == d.DGN_ERR_INVALID_ARG, n
    assert back(nb - 1) == d.DGN_ERR_WORKSPACE_TOO_SMALL
    for out in ("dx", "dweight", "dbias", "dstate0", "scratch"):
        for n in good:
            if n != out:
                assert back(**{out: good[n]}) == d.DGN_ERR_INVALID_ARG, (out, n)
    step = lambda n=4, slots=None, x=1 << 20, si=2 << 20, so=2 << 20, y=3 << 20, w=4 << 20: (  # noqa: E731
        d.dgn_conv_step(m, n, x, w, None, slots, si, so, y, stream=0))
    assert step(n=-1) == -1 and step(n=2**31) == -3 and step(x=0) == -2 and step(y=0) == -2 and step(w=0) == -2 and step(si=0) == -2
    assert step(slots=2) == -1 and step(y=2 << 20) == -1 and step(so=(2 << 20) + 24) == -1 and step(so=1 << 20) == -1
    assert step(y=(1 << 20) + 24) == -1 and step(y=4 << 20) == -1
    empty = conv_desc(d, num_channels=0)
    assert d.dgn_conv_forward(empty, *[None] * 8, 0, stream=0) == 0 and d.dgn_conv_backward(empty, *[None] * 12, 0, stream=0) == 0
    assert d.dgn_conv_forward(conv_desc(d, num_seqs=0), *[None] * 8, 0, stream=0) == 0
    assert d.dgn_conv_step(conv_desc(d, num_tokens=0), 3, *[None] * 7, stream=0) == 0


def test_select_description_is_checked(d):
    rc, sb, cb = d.dgn_select_workspace(select_desc(d))
    assert rc == 0 and sb > 0 and cb >= 12 * 5 * 4 and d.dgn_select_workspace(None)[0] == d.DGN_ERR_NULL_PTR
    for bad, code in [(dict(num_tokens=-1), -1), (dict(num_seqs=-1), -1), (dict(num_channels=-1), -1), (dict(num_states=0), -1),
                      (dict(num_groups=0), -1), (dict(num_groups=5), -1), (dict(dtype=-1), -1), (dict(x_stride=11), -1),
                      (dict(b_stride=14), -1), (dict(dc_stride=-15), -1), (dict(num_states=257), -3), (dict(num_tokens=2**31 - 1), -3),
                      (dict(num_seqs=2**31), -3), (dict(num_channels=3 * 2**30), -3), (dict(z_stride=2**41), -3)]:
        assert d.dgn_select_workspace(select_desc(d, **bad))[0] == code, bad
        assert d.dgn_select_step(select_desc(d, **bad), 4, d.dgn_select_inputs(), None, 64, 64, 64, stream=0) == code, bad
    assert d.dgn_select_workspace(select_desc(d, num_tokens=2**31 - 2, num_channels=2**15 * 3))[0] == d.DGN_ERR_TOO_LARGE


INPUTS = ("x", "delta", "A", "B", "C", "D", "delta_bias", "z", "seq_rowptr", "h0")
GRADS = ("dx", "ddelta", "dA", "dB", "dC", "dD", "ddelta_bias", "dz", "dh0")


def test_select_calls_refuse_bad_pointers(d):
    m = select_desc(d)
    _, nb, _ = d.dgn_select_workspace(m)
    good = apart(INPUTS + ("y", "final", "carry", "scratch"))

    def forward(scratch_bytes=nb, **kw):
        a = {**good, **kw}
        return d.dgn_select_forward(m, d.dgn_select_inputs(*(a[n] for n in INPUTS)), a["y"], a["final"], a["carry"], a["scratch"],
                                    scratch_bytes, stream=0)
    for n in ("x", "delta", "A", "B", "C", "seq_rowptr", "y", "scratch"):
        assert forward(**{n: None}) == d.DGN_ERR_NULL_PTR, n
    for n in good:
        assert forward(**{n: good[n] + 1}) == d.DGN_ERR_INVALID_ARG, n
    assert forward(nb - 1) == d.DGN_ERR_WORKSPACE_TOO_SMALL
    assert d.dgn_select_forward(m, None, 64, 64, 64, 64, nb, stream=0) == d.DGN_ERR_NULL_PTR
    for out in ("y", "final", "carry", "scratch"):
        for n in good:
            if n != out and (out, n) != ("final", "h0"):
                assert forward(**{out: good[n]}) == d.DGN_ERR_INVALID_ARG, (out, n)
    good = apart(INPUTS + ("carry", "dy", "dfinal") + GRADS + ("scratch",))

    def back(scratch_bytes=nb, **kw):
        a = {**good, **kw}
        return d.dgn_select_backward(m, d.dgn_select_inputs(*(a[n] for n in INPUTS)), a["carry"], a["dy"], a["dfinal"],
                                     d.dgn_select_grads(*(a[n] for n in GRADS)), a["scratch"], scratch_bytes, stream=0)
    for n in ("x", "delta", "A", "B", "C", "seq_rowptr", "carry", "dy", "dx", "ddelta", "dA", "dB", "dC", "dz", "scratch"):
        assert back(**{n: None}) == d.DGN_ERR_NULL_PTR, n
    for n in good:
        assert back(**{n: good[n] + 1}) == d.DGN_ERR_INVALID_ARG, n
    assert back(nb - 1) == d.DGN_ERR_WORKSPACE_TOO_SMALL
    for out in GRADS + ("scratch",):
        for n in good:
            if n != out:
                assert back(**{out: good[n]}) == d.DGN_ERR_INVALID_ARG, (out, n)
    good = apart(INPUTS[:8] + ("slots", "state_in", "state_out", "y"))

    def step(n=4, **kw):
        a = {**good, **kw}
        return d.dgn_select_step(m, n, d.dgn_select_inputs(*(a[k] for k in INPUTS[:8])), a["slots"], a["state_in"], a["state_out"], a["y"],
                                 stream=0)
    assert step(-1) == -1 and step(2**31) == -3
    for n in ("x", "delta", "A", "B", "C", "state_in", "state_out", "y"):
        assert step(**{n: None}) == d.DGN_ERR_NULL_PTR, n
    for n in good:
        assert step(**{n: good[n] + 1}) == d.DGN_ERR_INVALID_ARG, n
        for out in ("state_out", "y"):
            if n != out and not (out, n) in [("state_out", "state_in"), ("y", "x"), ("y", "delta"), ("y", "z")]:
                assert step(**{out: good[n]}) == d.DGN_ERR_INVALID_ARG, (out, n)
    assert step(state_out=good["state_in"] + 240) == -1 and step(y=good["x"] + 24) == -1
    for empty in (select_desc(d, num_channels=0), select_desc(d, num_seqs=0)):
        assert d.dgn_select_forward(empty, None, None, None, None, None, 0, stream=0) == 0
    assert d.dgn_select_backward(select_desc(d, num_channels=0), None, None, None, None, d.dgn_select_grads(), None, 0, stream=0) == 0
    assert d.dgn_select_step(select_desc(d, num_tokens=0), 3, None, None, None, None, None, stream=0) == 0


def test_dropout_is_checked(d):
    def call(x=1 << 20, r=2 << 20, key=3 << 20, y=4 << 20, **kw):
        m = d.dgn_dropout_desc(**{**dict(num_rows=5, num_columns=12, dtype=d.DGN_BF16, rate=0.5), **kw})
        return d.dgn_dropout(m, x, r, key, y, stream=0)
    for bad, code in [(dict(num_rows=-1), -1), (dict(num_columns=-1), -1), (dict(dtype=4), -1), (dict(rate=-0.1), -1), (dict(rate=1.5), -1),
                      (dict(rate=float("nan")), -1), (dict(x_stride=11), -1), (dict(y_stride=-1), -1), (dict(residual_stride=2**41), -3),
                      (dict(num_rows=2**31), -3), (dict(x=0), -2), (dict(key=0), -2), (dict(y=0), -2), (dict(x=(1 << 20) + 1), -1),
                      (dict(key=(3 << 20) + 4), -1), (dict(y=(1 << 20) + 2), -1), (dict(y=(2 << 20) + 24), -1), (dict(y=3 << 20), -1),
                      (dict(y=1 << 20, x_stride=13), -1)]:
        assert call(**bad) == code, bad
    assert d.dgn_dropout(None, 64, 64, 64, 64, stream=0) == d.DGN_ERR_NULL_PTR
    assert call(num_rows=0, x=0, y=0, key=0) == 0 and call(num_columns=0, x=0, y=0, key=0) == 0


def test_owners_refuse_before_they_allocate(d):
    for make in (lambda: d.ConvBuffers(4, 1, 8, taps=5), lambda: d.ConvBuffers(4, 1, 8, activation="gelu"),
                 lambda: d.ConvBuffers(4, 1, 8, dtype=torch.float64), lambda: d.ConvStepBuffers(4, 4, -8),
                 lambda: d.SelectiveBuffers(4, 1, 8, num_states=0), lambda: d.SelectiveBuffers(4, 1, 8, num_groups=3),
                 lambda: d.SelectiveStepBuffers(4, 4, 8, dtype=torch.int32), lambda: d.DropoutBuffers(4, 4, 1.5),
                 lambda: d.DropoutBuffers(4, -4, 0.5), lambda: d.DropoutBuffers(4, 4, 0.5, dtype=torch.float64)):
        with pytest.raises(d.DgnError):
            make()
    for make in (lambda: d.ConvBuffers(4, 1, 8, device="cpu"), lambda: d.ConvStepBuffers(4, 4, 8, device="cpu"),
                 lambda: d.SelectiveBuffers(4, 1, 8, device="cpu"), lambda: d.SelectiveStepBuffers(4, 4, 8, device="cpu"),
                 lambda: d.DropoutBuffers(4, 4, 0.5, device="cpu")):
        with pytest.raises(d.DgnError):
            make()


def differences(plain, inputs, dy, dfinal, prefix="d"):
    """The gradients of a plain form against central differences of its own loss, in a random direction each."""
    gen = torch.Generator().manual_seed(9)

    def loss(i):
        r = plain(**i)
        return float((r["y"][0] * dy).sum() + (r["final"][0] * dfinal).sum())
    grads = plain(**inputs, dy=dy, dfinal=dfinal)
    for n in inputs:
        way = torch.randn(inputs[n].shape, generator=gen, dtype=torch.float64)
        up, down = ({**inputs, n: inputs[n] + s * way} for s in (1e-5, -1e-5))
        got = float((grads[prefix + n][0] * way).sum())
        assert abs((loss(up) - loss(down)) / 2e-5 - got) < 1e-6 * (1 + abs(got)), n


def test_the_plain_forms_agree_with_their_differences():
    gen = torch.Generator().manual_seed(3)
    rn = lambda *s: torch.randn(*s, generator=gen, dtype=torch.float64)  # noqa: E731
    ptr = torch.tensor([0, 4, 4, 11, 12])
    for act in ("none", "silu"):
        differences(lambda **i: lo.conv(rowptr=ptr, act=act, **i), dict(x=rn(12, 3), weight=rn(3, 4), bias=rn(3), state0=rn(4, 3, 3)),
                    rn(12, 3), rn(4, 3, 3))
    c, n, g = 6, 3, 2
    differences(lambda **i: lo.select(rowptr=ptr, groups=g, **i),
                dict(x=rn(12, c), delta=rn(12, c), A=-torch.exp(rn(c, n)), B=rn(12, g * n), C=rn(12, g * n), D=rn(c), delta_bias=rn(c),
                     z=rn(12, c), h0=rn(4, c, n)), rn(12, c), rn(4, c, n))


def test_the_generator_gives_the_published_numbers():
    """Known answers that its authors publish with it (ten rounds, four words)."""
    assert lo.philox((0, 0, 0, 0), (0, 0)) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    ones = 0xFFFFFFFF
    assert lo.philox((ones, ones, ones, ones), (ones, ones)) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    assert np.array_equal(lo.draws(16, 0, 0)[:8], [0xE8D5, 0x6627, 0xC58D, 0xE169, 0xAC4C, 0xBC57, 0xDBD8, 0x9B00])


def test_the_largest_scans_fit_one_launch_with_the_empty_sequences(d):
    """A launch of less than 2^32 threads has the strips' workgroups of 256 and up to 1 024 more, for states of sequences without rows."""
    one = lambda groups_: select_desc(d, num_tokens=64 * groups_, num_channels=1, num_groups=1, num_states=16)  # noqa: E731
    assert d.dgn_select_workspace(one(2**24 - 1025))[0] == 0
    for strips in (2**24 - 1024, 2**24 - 1000, 2**24 - 1):
        assert d.dgn_select_workspace(one(strips))[0] == d.DGN_ERR_TOO_LARGE, strips


def test_the_widest_convolutions_fit_one_launch(d):
    """The sums of a tap take a workgroup of 1 024 threads for 64 channels, in launches of less than 2^32 threads."""
    for dtype in (d.DGN_F32, d.DGN_BF16):
        wide = lambda c: conv_desc(d, num_tokens=1, num_channels=c, dtype=dtype)  # noqa: E731
        assert d.dgn_conv_workspace(wide(2**28 - 64))[0] == 0
        for c in (2**28 - 63, 2**28 - 1):
            assert d.dgn_conv_workspace(wide(c))[0] == d.DGN_ERR_TOO_LARGE, c


def test_scans_without_gradients_ask_for_the_forward_pass_alone(d):
    """The states of the strips, their sums of steps, and a copy of h0; no carry.  What is refused then."""
    for states, gib in ((16, 0.07), (64, 0.28), (128, 0.56), (256, 1.1)):
        m = dict(num_tokens=16384, num_seqs=8, num_channels=2048, num_states=states, num_groups=1)
        rc, need, carry = d.dgn_select_workspace(select_desc(d, **m, forward_only=1))
        both = d.dgn_select_workspace(select_desc(d, **m))
        assert rc == 0 and carry == 0 and need < gib * 2**30 and both[0] == 0 and both[1] >= need and both[2] > 0, (states, need)
    assert d.dgn_select_workspace(select_desc(d, forward_only=2))[0] == d.DGN_ERR_INVALID_ARG
    m = select_desc(d, forward_only=1)
    need, good = d.dgn_select_workspace(m)[1], apart(INPUTS + ("y", "final", "carry", "scratch"))
    inputs = d.dgn_select_inputs(*(good[n] for n in INPUTS))
    assert d.dgn_select_forward(m, inputs, good["y"], good["final"], good["carry"], good["scratch"], need, stream=0) == d.DGN_ERR_INVALID_ARG
    assert d.dgn_select_forward(m, inputs, good["y"], good["final"], None, good["scratch"], need - 1, stream=0) == d.DGN_ERR_WORKSPACE_TOO_SMALL
    grads = d.dgn_select_grads(*(64 for _ in GRADS))
    assert d.dgn_select_backward(m, inputs, good["carry"], 64, None, grads, good["scratch"], 2**30, stream=0) == d.DGN_ERR_INVALID_ARG


def test_the_scratch_of_scans_grows_with_the_states_and_not_with_their_square(d):
    """The gradients' sums over channels go through a buffer of 256 MiB, or of some thousand workgroups' rows; the rest is three states a strip."""
    for states, gib in ((64, 0.7), (128, 1.4), (256, 2.6)):
        m = select_desc(d, num_tokens=16384, num_seqs=8, num_channels=2048, num_states=states, num_groups=1)
        rc, need, _ = d.dgn_select_workspace(m)
        assert rc == 0 and need < gib * 2**30, (states, need / 2**30)
