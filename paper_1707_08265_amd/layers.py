"""Owners of buffers for the operators of a selective recurrent layer: the short causal convolution, the selective scan, and
dropout that is added to a residual.  Checks, errors, streams and devices are as in ``values``: allocation, checks of types and
shapes, and marshalling only; calls on one owner share its outputs and scratch.
"""
from __future__ import annotations

import ctypes

import torch

from . import binding as b
from .values import DTYPES, _dense, _need, _queue, _rows, _strides

ACTIVATIONS = {"none": b.DGN_ACT_NONE, "silu": b.DGN_ACT_SILU}


def _conv_desc(tokens, seqs, channels, taps, activation, dtype):
    _need(activation in ACTIVATIONS and dtype in DTYPES, "activation or element type")
    return b.dgn_conv_desc(num_tokens=tokens, num_seqs=seqs, num_channels=channels, num_taps=taps,
                           activation=ACTIVATIONS[activation], dtype=DTYPES[dtype])


class ConvBuffers:
    """Outputs and scratch of the short causal convolution over ``num_seqs`` sequences in ``num_tokens`` rows.

    ``forward`` writes ``y`` and ``final``, the last ``taps - 1`` rows of each sequence; with ``train``, ``backward``, given the
    same inputs, writes ``dx``, ``dweight``, ``dbias`` and ``dstate0``."""

    def __init__(self, num_tokens, num_seqs, num_channels, taps=4, activation="silu", dtype=torch.bfloat16, train=False,
                 device="cuda"):
        self._d = _conv_desc(num_tokens, num_seqs, num_channels, taps, activation, dtype)
        rc, sb = b.dgn_conv_workspace(self._d)
        b._check(rc, "dgn_conv_workspace")
        self.num_tokens, self.num_seqs, self.num_channels = num_tokens, num_seqs, num_channels
        self.taps, self.dtype, self.train = taps, dtype, bool(train)
        self._wide, self._ptr, self._states = (num_tokens, num_channels), (num_seqs + 1,), (num_seqs, taps - 1, num_channels)
        self._weight, self._one = (num_channels, taps), (num_channels,)
        new = lambda shape, dtype=dtype: torch.zeros(shape, dtype=dtype, device=device)  # noqa: E731
        self.y, self.final = new(self._wide), new(self._states)
        self.device, self._index = self.y.device, self.y.get_device()
        _need(self._index >= 0, "device: not a GPU")
        self._scratch, self._scratch_bytes = torch.empty(sb, dtype=torch.uint8, device=device), sb
        if train:
            self.dx, self.dstate0 = new(self._wide), new(self._states)
            self.dweight, self.dbias = new(self._weight, torch.float32), new(self._one, torch.float32)

    def _inputs(self, x, weight, seq_rowptr, bias, state0):
        at = self._index
        px, sx = _rows(x, self._wide, self.dtype, at, "x")
        return (px, sx, _dense(weight, self._weight, torch.float32, at, "weight"), _dense(bias, self._one, torch.float32, at, "bias"),
                _dense(seq_rowptr, self._ptr, torch.int64, at, "seq_rowptr"), _dense(state0, self._states, self.dtype, at, "state0"))

    def forward(self, x, weight, seq_rowptr, bias=None, state0=None, stream=None):
        """``x`` [tokens, channels], ``weight`` float [channels, taps], ``bias`` float [channels], ``seq_rowptr`` int64 [seqs + 1],
        ``state0`` [seqs, taps - 1, channels]: may be ``final`` itself, for sequences that go on from call to call."""
        px, sx, pw, pb, pr, ps = self._inputs(x, weight, seq_rowptr, bias, state0)
        d = self._d = _strides(self._d, x_stride=sx)
        b._check(b._lib.dgn_conv_forward(ctypes.byref(d), px, pw, pb, pr, ps, self.y.data_ptr(), self.final.data_ptr(),
                                         self._scratch.data_ptr(), self._scratch_bytes, _queue(self._index, stream)),
                 "dgn_conv_forward")

    def backward(self, x, weight, seq_rowptr, dy, bias=None, state0=None, dfinal=None, stream=None):
        """Gradients for ``dy`` [tokens, channels] and ``dfinal`` [seqs, taps - 1, channels].  ``state0`` may not be ``final``, where
        ``forward`` has written since."""
        _need(self.train, "backward of buffers made without train")
        px, sx, pw, pb, pr, ps = self._inputs(x, weight, seq_rowptr, bias, state0)
        if ps:
            _need(abs(ps - self.final.data_ptr()) >= self.final.nbytes, "state0 of backward: final has been written")
        py, sy = _rows(dy, self._wide, self.dtype, self._index, "dy")
        d = self._d = _strides(self._d, x_stride=sx, dy_stride=sy)
        pf = _dense(dfinal, self._states, self.dtype, self._index, "dfinal")
        b._check(b._lib.dgn_conv_backward(ctypes.byref(d), px, pw, pb, pr, ps, py, pf, self.dx.data_ptr(), self.dweight.data_ptr(),
                                          self.dbias.data_ptr(), self.dstate0.data_ptr(), self._scratch.data_ptr(),
                                          self._scratch_bytes, _queue(self._index, stream)), "dgn_conv_backward")


class ConvStepBuffers:
    """Output of one token of the convolution for each of ``num_rows`` rows, on states in a pool of ``num_slots``."""

    def __init__(self, num_rows, num_slots, num_channels, taps=4, activation="silu", dtype=torch.bfloat16, device="cuda"):
        self._d = _conv_desc(num_rows, 0, num_channels, taps, activation, dtype)
        b._check(b.dgn_conv_workspace(self._d)[0], "dgn_conv_workspace")
        self.num_rows, self.num_slots, self.num_channels, self.taps, self.dtype = num_rows, num_slots, num_channels, taps, dtype
        self._wide, self._slots, self._pool = (num_rows, num_channels), (num_rows,), (num_slots, taps - 1, num_channels)
        self._weight, self._one = (num_channels, taps), (num_channels,)
        self.y = torch.empty(self._wide, dtype=dtype, device=device)
        self.device, self._index = self.y.device, self.y.get_device()
        _need(self._index >= 0, "device: not a GPU")

    def step(self, x, weight, slots, state_in, state_out=None, bias=None, stream=None):
        """Row r takes the rows before it from row ``slots[r]`` of ``state_in`` [slots, taps - 1, channels] and leaves them, moved on
        by one, in the same row of ``state_out`` (default: ``state_in`` itself).  ``slots``: int32, -1 for an idle row, or None: row r."""
        at = self._index
        px, sx = _rows(x, self._wide, self.dtype, at, "x")
        d = self._d = _strides(self._d, x_stride=sx)
        pi = _dense(state_in, self._pool, self.dtype, at, "state_in")
        po = pi if state_out is None else _dense(state_out, self._pool, self.dtype, at, "state_out")
        b._check(b._lib.dgn_conv_step(ctypes.byref(d), self.num_slots, px, _dense(weight, self._weight, torch.float32, at, "weight"),
                                      _dense(bias, self._one, torch.float32, at, "bias"),
                                      _dense(slots, self._slots, torch.int32, at, "slots"), pi, po, self.y.data_ptr(),
                                      _queue(at, stream)), "dgn_conv_step")


def _select_desc(tokens, seqs, channels, states, groups, dtype, train):
    _need(dtype in DTYPES, "element type")
    return b.dgn_select_desc(num_tokens=tokens, num_seqs=seqs, num_channels=channels, num_states=states, num_groups=groups,
                             dtype=DTYPES[dtype], forward_only=0 if train else 1)


class _Selective:
    """What the scan and its step share: sizes, and the checks of the inputs."""

    def _sizes(self, rows, channels, states, groups, dtype, device):
        self.num_channels, self.num_states, self.num_groups, self.dtype = channels, states, groups, dtype
        self._wide, self._shared, self._params, self._one = (rows, channels), (rows, groups * states), (channels, states), (channels,)
        self.y = torch.zeros(self._wide, dtype=dtype, device=device)        # (rows of no sequence are not written)
        self.device, self._index = self.y.device, self.y.get_device()
        _need(self._index >= 0, "device: not a GPU")

    def _inputs(self, x, delta, A, B, C, D, delta_bias, z, seq_rowptr=None, h0=None, **strides):
        at, wide, dtype, f32 = self._index, self._wide, self.dtype, torch.float32
        px, sx = _rows(x, wide, dtype, at, "x")
        pd, sd = _rows(delta, wide, dtype, at, "delta")
        pb, sb = _rows(B, self._shared, dtype, at, "B")
        pc, sc = _rows(C, self._shared, dtype, at, "C")
        pz, sz = (None, self._d.z_stride) if z is None else _rows(z, wide, dtype, at, "z")
        d = self._d = _strides(self._d, x_stride=sx, delta_stride=sd, b_stride=sb, c_stride=sc, z_stride=sz, **strides)
        return d, b.dgn_select_inputs(px, pd, _dense(A, self._params, f32, at, "A"), pb, pc, _dense(D, self._one, f32, at, "D"),
                                      _dense(delta_bias, self._one, f32, at, "delta_bias"), pz, seq_rowptr, h0)


class SelectiveBuffers(_Selective):
    """Outputs and scratch of the selective scan over ``num_seqs`` sequences in ``num_tokens`` rows.

    ``forward`` writes ``y`` and ``final``; with ``train`` it keeps the states that ``backward`` starts from, and ``backward``, given
    the same inputs, writes ``dx``, ``ddelta``, ``dA``, ``dB``, ``dC``, ``dD``, ``ddelta_bias``, ``dz`` and ``dh0``."""

    def __init__(self, num_tokens, num_seqs, num_channels, num_states=16, num_groups=1, dtype=torch.bfloat16, train=False,
                 device="cuda"):
        self._d = _select_desc(num_tokens, num_seqs, num_channels, num_states, num_groups, dtype, train)
        rc, sb, cb = b.dgn_select_workspace(self._d)
        b._check(rc, "dgn_select_workspace")
        self._sizes(num_tokens, num_channels, num_states, num_groups, dtype, device)
        self.num_tokens, self.num_seqs, self.train = num_tokens, num_seqs, bool(train)
        self._ptr, self._states = (num_seqs + 1,), (num_seqs, num_channels, num_states)
        new = lambda shape, dtype=torch.float32: torch.zeros(shape, dtype=dtype, device=device)  # noqa: E731
        self.final = new(self._states)
        self._scratch, self._scratch_bytes = torch.empty(sb, dtype=torch.uint8, device=device), sb
        self._carry = torch.empty(cb, dtype=torch.uint8, device=device) if train else None
        if train:
            self.dx, self.ddelta, self.dz = new(self._wide, dtype), new(self._wide, dtype), new(self._wide, dtype)
            self.dB, self.dC = new(self._shared, dtype), new(self._shared, dtype)
            self.dA, self.dD, self.ddelta_bias, self.dh0 = new(self._params), new(self._one), new(self._one), new(self._states)
            self._grads = b.dgn_select_grads(*(t.data_ptr() for t in (self.dx, self.ddelta, self.dA, self.dB, self.dC, self.dD,
                                                                      self.ddelta_bias, self.dz, self.dh0)))

    def _starts(self, seq_rowptr, h0):
        return (_dense(seq_rowptr, self._ptr, torch.int64, self._index, "seq_rowptr"),
                _dense(h0, self._states, torch.float32, self._index, "h0"))

    def forward(self, x, delta, A, B, C, seq_rowptr, D=None, delta_bias=None, z=None, h0=None, stream=None):
        """``x``, ``delta``, ``z`` [tokens, channels], ``A`` float [channels, states], ``B``, ``C`` [tokens, groups * states], ``D``,
        ``delta_bias`` float [channels], ``seq_rowptr`` int64 [seqs + 1], ``h0`` float [seqs, channels, states]: may be ``final``
        itself, for sequences that go on from call to call."""
        pr, ph = self._starts(seq_rowptr, h0)
        d, inputs = self._inputs(x, delta, A, B, C, D, delta_bias, z, pr, ph)
        b._check(b._lib.dgn_select_forward(ctypes.byref(d), ctypes.byref(inputs), self.y.data_ptr(), self.final.data_ptr(),
                                           b._dp(self._carry), self._scratch.data_ptr(), self._scratch_bytes,
                                           _queue(self._index, stream)), "dgn_select_forward")

    def backward(self, x, delta, A, B, C, seq_rowptr, dy, D=None, delta_bias=None, z=None, h0=None, dfinal=None, stream=None):
        """Gradients for ``dy`` [tokens, channels] and ``dfinal`` float [seqs, channels, states] of the last ``forward``.  ``h0`` may not
        be ``final``, where ``forward`` has written since.  Without ``z``, ``dz`` is left as it is."""
        _need(self.train, "backward of buffers made without train")
        pr, ph = self._starts(seq_rowptr, h0)
        if ph:
            _need(abs(ph - self.final.data_ptr()) >= self.final.nbytes, "h0 of backward: final has been written")
        py, sy = _rows(dy, self._wide, self.dtype, self._index, "dy")
        d, inputs = self._inputs(x, delta, A, B, C, D, delta_bias, z, pr, ph, dy_stride=sy)
        pf = _dense(dfinal, self._states, torch.float32, self._index, "dfinal")
        b._check(b._lib.dgn_select_backward(ctypes.byref(d), ctypes.byref(inputs), b._dp(self._carry), py, pf,
                                            ctypes.byref(self._grads), self._scratch.data_ptr(), self._scratch_bytes,
                                            _queue(self._index, stream)), "dgn_select_backward")


class SelectiveStepBuffers(_Selective):
    """Output of one token of the selective scan for each of ``num_rows`` rows, on states in a pool of ``num_slots``."""

    def __init__(self, num_rows, num_slots, num_channels, num_states=16, num_groups=1, dtype=torch.bfloat16, device="cuda"):
        self._d = _select_desc(num_rows, 0, num_channels, num_states, num_groups, dtype, False)
        b._check(b.dgn_select_workspace(self._d)[0], "dgn_select_workspace")
        self._sizes(num_rows, num_channels, num_states, num_groups, dtype, device)
        self.num_rows, self.num_slots = num_rows, num_slots
        self._slots, self._pool = (num_rows,), (num_slots, num_channels, num_states)

    def step(self, x, delta, A, B, C, slots, state_in, state_out=None, D=None, delta_bias=None, z=None, stream=None):
        """Row r takes its states from row ``slots[r]`` of ``state_in`` (float [slots, channels, states]) and leaves them in the same
        row of ``state_out`` (default: ``state_in`` itself).  ``slots``: int32, -1 for an idle row, or None: row r."""
        at = self._index
        d, inputs = self._inputs(x, delta, A, B, C, D, delta_bias, z)
        pi = _dense(state_in, self._pool, torch.float32, at, "state_in")
        po = pi if state_out is None else _dense(state_out, self._pool, torch.float32, at, "state_out")
        b._check(b._lib.dgn_select_step(ctypes.byref(d), self.num_slots, ctypes.byref(inputs),
                                        _dense(slots, self._slots, torch.int32, at, "slots"), pi, po, self.y.data_ptr(),
                                        _queue(at, stream)), "dgn_select_step")


class DropoutBuffers:
    """Outputs of dropout, at ``rate``, of ``num_rows`` rows that are added to a residual, and its gradient.

    ``key``: int64 [2] on the GPU, a seed and the number of the step.  It is read when a call runs; both passes of a step take the
    same one, and the next step another (``key[1] += 1``, also between replays of a captured graph)."""

    def __init__(self, num_rows, num_columns, rate, dtype=torch.bfloat16, device="cuda"):
        _need(dtype in DTYPES, "element type")
        self._d = b.dgn_dropout_desc(num_rows=num_rows, num_columns=num_columns, dtype=DTYPES[dtype], rate=rate)
        _need(num_rows >= 0 and num_columns >= 0 and 0.0 <= rate <= 1.0, "dropout: sizes or rate")
        self.rate, self.dtype, self._wide = rate, dtype, (num_rows, num_columns)
        self.y, self.dx = (torch.empty(self._wide, dtype=dtype, device=device) for _ in range(2))
        self.device, self._index = self.y.device, self.y.get_device()
        _need(self._index >= 0, "device: not a GPU")

    def _drop(self, x, residual, key, out, stream):
        at = self._index
        px, sx = _rows(x, self._wide, self.dtype, at, "x")
        pr, sr = (None, self._d.residual_stride) if residual is None else _rows(residual, self._wide, self.dtype, at, "residual")
        d = self._d = _strides(self._d, x_stride=sx, residual_stride=sr)
        b._check(b._lib.dgn_dropout(ctypes.byref(d), px, pr, _dense(key, (2,), torch.int64, at, "key"), out.data_ptr(),
                                    _queue(at, stream)), "dgn_dropout")

    def forward(self, x, key, residual=None, stream=None):
        """``y`` = ``residual`` + ``x``, dropped and scaled; both [rows, columns]."""
        self._drop(x, residual, key, self.y, stream)

    def backward(self, dy, key, stream=None):
        """``dx``, for ``dy`` [rows, columns]; the residual's gradient is ``dy`` itself."""
        self._drop(dy, None, key, self.dx, stream)
