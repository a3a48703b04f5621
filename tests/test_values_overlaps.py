"""Memory that a call writes must not be what it reads elsewhere: refused before any device work.  (Addresses here are numbers.)"""
import pytest

import paper_1707_08265_amd as d

N, C, SEQS = 10, 12, 2                      # 10 rows of 12 channels in bf16: 240 bytes; states 96 bytes; row pointers 24
STEP = 1 << 12
NAMES = ["x", "gate", "rowptr", "h0", "y", "final", "carry", "scratch", "dy", "dfinal", "dx", "dgate", "dh0"]
APART = {name: STEP * (i + 1) for i, name in enumerate(NAMES)}


def desc(**kw):
    return d.dgn_scan_desc(**{**dict(num_tokens=N, num_seqs=SEQS, num_channels=C, gate_group=1, dtype=d.DGN_BF16,
                                     gate_kind=d.DGN_GATE_DECAY), **kw})


def forward(m=None, **at):
    a = {**APART, **at}
    return d.dgn_scan_forward(m or desc(), *(a[n] for n in ("x", "gate", "rowptr", "h0", "y", "final", "carry", "scratch")), 1 << 20,
                              stream=0)


def backward(m=None, **at):
    a = {**APART, **at}
    return d.dgn_scan_backward(m or desc(), *(a[n] for n in ("x", "gate", "rowptr", "h0", "carry", "dy", "dfinal", "dx", "dgate", "dh0",
                                                             "scratch")), 1 << 20, stream=0)


def step(m=None, **at):
    a = {**dict(x=STEP, gate=2 * STEP, slots=3 * STEP, state_in=4 * STEP, state_out=4 * STEP, y=5 * STEP), **at}
    return d.dgn_scan_step(m or desc(), 8, *(a[n] for n in ("x", "gate", "slots", "state_in", "state_out", "y")), stream=0)


def test_forward():
    for out, others in [("y", ("x", "gate", "rowptr", "h0", "final")), ("final", ("x", "gate", "rowptr"))]:
        for other in others:
            for off in (0, 8, 16):
                assert forward(**{out: APART[other] + off}) == d.DGN_ERR_INVALID_ARG, (out, other, off)
    assert forward(y=APART["x"] + 238) == forward(y=APART["x"] - 238) == d.DGN_ERR_INVALID_ARG      # the last and the first element


def test_backward():
    for out in ("dx", "dgate", "dh0"):
        for other in ("x", "gate", "rowptr", "h0", "dy", "dfinal", "dx", "dgate"):
            if out == other or (out, other) == ("dh0", "dfinal"):
                continue
            for off in (0, 8, 16):
                if (out, other, off) != ("dh0", "h0", 0):
                    assert backward(**{out: APART[other] + off}) == d.DGN_ERR_INVALID_ARG, (out, other, off)


def test_one_token():
    for bad in [dict(y=4 * STEP), dict(y=3 * STEP), dict(y=STEP + 2), dict(y=2 * STEP - 2), dict(state_out=4 * STEP + 48), dict(state_out=STEP),
                dict(state_out=3 * STEP), dict(state_out=5 * STEP)]:
        assert step(**bad) == d.DGN_ERR_INVALID_ARG, bad
    assert step(desc(gate_group=3), y=2 * STEP) == d.DGN_ERR_INVALID_ARG                            # a gate of other channels
    assert step(desc(x_stride=20), y=STEP) == d.DGN_ERR_INVALID_ARG


@pytest.mark.parametrize("off", [2, 22, 24 + 78, 78])
def test_columns_of_one_matrix_that_meet(off):
    """Rows 80 bytes apart, 24 wide: columns that begin 2, 22 or -2 bytes from the others'."""
    assert forward(desc(x_stride=40, y_stride=40), y=APART["x"] + off) == d.DGN_ERR_INVALID_ARG


def test_rows_of_which_nobody_knows():
    assert forward(desc(x_stride=40, y_stride=41), y=APART["x"] + 24) == d.DGN_ERR_INVALID_ARG
    huge = desc(num_channels=2**31 - 2, x_stride=2**40)
    assert d.dgn_scan_step(huge, 2**31 - 2, 2, 2, None, 4, 8, 2, stream=0) == d.DGN_ERR_INVALID_ARG
