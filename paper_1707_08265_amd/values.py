"""Owners of buffers for the operators on tensor values: the gated linear recurrence, and lists of tensors with their
norms, clipping and update.  Allocation, checks of types and shapes, and marshalling only.

The library sees addresses; what a tensor's type, shape and strides say is checked here.  Every method raises
``DgnError`` for what is refused, by these checks or by the library.  Kernels run on the current stream, or on
``stream``; a caller who uses another stream than the one its tensors belong to orders the two, as for any kernel.
Calls on one owner share its outputs and scratch: they must not overlap, whether from several streams or host threads.
"""
from __future__ import annotations

import ctypes

import numpy as np
import torch

from . import binding as b

DTYPES = {torch.float32: b.DGN_F32, torch.float16: b.DGN_F16, torch.bfloat16: b.DGN_BF16}
GATES = {"decay": b.DGN_GATE_DECAY, "sigmoid": b.DGN_GATE_SIGMOID}


_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _need(ok, where):
    if not ok:
        raise b.DgnError(b.DGN_ERR_INVALID_ARG, where)


def _queue(index, stream):
    """The stream to launch on: the current one, or ``stream``.  It and the current device have to be of GPU ``index``."""
    if _current_device() != index or (stream is not None and isinstance(stream, torch.cuda.Stream) and stream.device_index != index):
        raise b.DgnError(b.DGN_ERR_INVALID_ARG, "the current device or stream is not of the buffers' GPU")
    return b._raw_stream(index) if stream is None and b._raw_stream is not None else b._stream(stream)


def _rows(t, shape, dtype, index, where):
    """Address and row stride of a matrix on GPU ``index`` whose rows have no gaps inside.  (Few questions to a tensor, each
    costs 50 to 200 ns: a call for a few tokens is as long as what is asked here and its launch.)"""
    if not isinstance(t, torch.Tensor) or t.dtype is not dtype or t.shape != shape or t.get_device() != index:
        raise b.DgnError(b.DGN_ERR_INVALID_ARG, where)
    rows, width = shape
    step, inner = t.stride()
    if (inner != 1 and width > 1) or (step < width and rows > 1):
        raise b.DgnError(b.DGN_ERR_INVALID_ARG, where)
    return t.data_ptr(), step if rows > 1 else 0


def _dense(t, shape, dtype, index, where):
    if t is None:
        return None
    if (not isinstance(t, torch.Tensor) or t.dtype is not dtype or t.shape != shape or t.get_device() != index
            or not t.is_contiguous()):
        raise b.DgnError(b.DGN_ERR_INVALID_ARG, where)
    return t.data_ptr()


def _strides(d, **strides):
    """The description ``d`` with these row strides: itself, if it has them, else another (a call may still read ``d``)."""
    for name, value in strides.items():
        if getattr(d, name) != value:
            d = type(d).from_buffer_copy(d)
            for name, value in strides.items():
                setattr(d, name, value)
            break
    return d


def _desc(tokens, seqs, channels, group, kind, dtype):
    _need(kind in GATES and dtype in DTYPES, "gate kind or element type")
    return b.dgn_scan_desc(num_tokens=tokens, num_seqs=seqs, num_channels=channels, gate_group=group,
                           dtype=DTYPES[dtype], gate_kind=GATES[kind])


class ScanBuffers:
    """Outputs and scratch of the gated linear recurrence over ``num_seqs`` sequences in ``num_tokens`` rows.

    ``forward`` writes ``y`` and ``final``; with ``train`` it keeps the states that ``backward`` starts from, and
    ``backward``, given the same inputs, writes ``dx``, ``dgate`` and ``dh0``.  ``gate_group`` channels share a gate."""

    def __init__(self, num_tokens, num_seqs, num_channels, gate_group=1, kind="sigmoid", dtype=torch.bfloat16,
                 train=False, device="cuda"):
        self._d = _desc(num_tokens, num_seqs, num_channels, gate_group, kind, dtype)
        rc, sb, cb = b.dgn_scan_workspace(self._d)
        b._check(rc, "dgn_scan_workspace")
        self.num_tokens, self.num_seqs, self.num_channels = num_tokens, num_seqs, num_channels
        self.num_heads, self.dtype, self.train = num_channels // gate_group, dtype, bool(train)
        # rows that belong to no sequence are not written: zero until they are
        new = lambda *shape, dtype=dtype: torch.zeros(shape, dtype=dtype, device=device)  # noqa: E731
        self.y = new(num_tokens, num_channels)
        self.final = new(num_seqs, num_channels, dtype=torch.float32)
        self.device, self._index = self.y.device, self.y.get_device()
        _need(self._index >= 0, "device: not a GPU")
        self._wide, self._gates = (num_tokens, num_channels), (num_tokens, self.num_heads)
        self._ptr, self._states = (num_seqs + 1,), (num_seqs, num_channels)
        self._scratch, self._scratch_bytes = torch.empty(sb, dtype=torch.uint8, device=device), sb
        self._carry = torch.empty(cb, dtype=torch.uint8, device=device) if train else None
        if train:
            self.dx, self.dgate = new(num_tokens, num_channels), new(num_tokens, self.num_heads)
            self.dh0 = new(num_seqs, num_channels, dtype=torch.float32)

    def _inputs(self, x, gate, seq_rowptr, h0):
        at = self._index
        px, sx = _rows(x, self._wide, self.dtype, at, "x")
        pg, sg = _rows(gate, self._gates, self.dtype, at, "gate")
        pr = _dense(seq_rowptr, self._ptr, torch.int64, at, "seq_rowptr")
        return px, sx, pg, sg, pr, _dense(h0, self._states, torch.float32, at, "h0")

    def forward(self, x, gate, seq_rowptr, h0=None, stream=None):
        """``x`` [tokens, channels], ``gate`` [tokens, heads], ``seq_rowptr`` int64 [seqs + 1], ``h0`` float [seqs, channels]:
        may be ``final`` itself, for sequences that go on from call to call."""
        px, sx, pg, sg, pr, ph = self._inputs(x, gate, seq_rowptr, h0)
        d = self._d = _strides(self._d, x_stride=sx, gate_stride=sg)
        b._check(b._lib.dgn_scan_forward(ctypes.byref(d), px, pg, pr, ph, self.y.data_ptr(), self.final.data_ptr(),
                                         b._dp(self._carry), self._scratch.data_ptr(), self._scratch_bytes,
                                         _queue(self._index, stream)), "dgn_scan_forward")

    def backward(self, x, gate, seq_rowptr, dy, h0=None, dfinal=None, stream=None):
        """Gradients for ``dy`` [tokens, channels] and ``dfinal`` float [seqs, channels] of the last ``forward``.  ``dfinal`` may be
        ``dh0``; ``h0`` may not be ``final``, where ``forward`` has written since."""
        _need(self.train, "backward of buffers made without train")
        px, sx, pg, sg, pr, ph = self._inputs(x, gate, seq_rowptr, h0)
        if ph:
            _need(abs(ph - self.final.data_ptr()) >= 4 * self.num_seqs * self.num_channels, "h0 of backward: final has been written")
        py, sy = _rows(dy, self._wide, self.dtype, self._index, "dy")
        d = self._d = _strides(self._d, x_stride=sx, gate_stride=sg, dy_stride=sy)
        pf = _dense(dfinal, self._states, torch.float32, self._index, "dfinal")
        b._check(b._lib.dgn_scan_backward(ctypes.byref(d), px, pg, pr, ph, b._dp(self._carry), py, pf,
                                          self.dx.data_ptr(), self.dgate.data_ptr(), self.dh0.data_ptr(),
                                          self._scratch.data_ptr(), self._scratch_bytes, _queue(self._index, stream)),
                 "dgn_scan_backward")


class ScanStepBuffers:
    """Output of one token of the recurrence for each of ``num_rows`` rows, on states in a pool of ``num_slots``."""

    def __init__(self, num_rows, num_slots, num_channels, gate_group=1, kind="sigmoid", dtype=torch.bfloat16, device="cuda"):
        self._d = _desc(num_rows, 0, num_channels, gate_group, kind, dtype)
        b._check(b.dgn_scan_workspace(self._d)[0], "dgn_scan_workspace")
        self.num_rows, self.num_slots, self.num_channels = num_rows, num_slots, num_channels
        self.num_heads, self.dtype = num_channels // gate_group, dtype
        self.y = torch.empty(num_rows, num_channels, dtype=dtype, device=device)
        self.device, self._index = self.y.device, self.y.get_device()
        _need(self._index >= 0, "device: not a GPU")
        self._wide, self._gates = (num_rows, num_channels), (num_rows, self.num_heads)
        self._one, self._pool = (num_rows,), (num_slots, num_channels)

    def step(self, x, gate, slots, state_in, state_out=None, stream=None):
        """Row r takes its state from row ``slots[r]`` of ``state_in`` (float [slots, channels]) and leaves it in the same
        row of ``state_out`` (default: ``state_in`` itself).  ``slots``: int32, -1 for an idle row, or None: row r."""
        at = self._index
        px, sx = _rows(x, self._wide, self.dtype, at, "x")
        pg, sg = _rows(gate, self._gates, self.dtype, at, "gate")
        d = self._d = _strides(self._d, x_stride=sx, gate_stride=sg)
        ps = _dense(slots, self._one, torch.int32, at, "slots")
        pi = _dense(state_in, self._pool, torch.float32, at, "state_in")
        po = pi if state_out is None else _dense(state_out, self._pool, torch.float32, at, "state_out")
        b._check(b._lib.dgn_scan_step(ctypes.byref(d), self.num_slots, px, pg, ps, pi, po, self.y.data_ptr(), _queue(self._index, stream)),
                 "dgn_scan_step")


class TensorList:
    """A list of contiguous tensors of one device whose addresses the library holds; keeps the tensors and their memory alive.

    The addresses are those of the tensors when the list is made.  A tensor that is given other memory later (``t.data = ...``,
    gradients that a framework allocates anew) needs a new list; the old one goes on with the old memory.  Making a list asks
    every tensor a few questions, copies a table and waits for the stream (2 000 tensors 0.8 ms), so gradients are best left
    where they are."""

    def __init__(self, tensors, stream=None):
        self.tensors = list(tensors)
        n = len(self.tensors)
        _need(n == 0 or isinstance(self.tensors[0], torch.Tensor), "TensorList")
        dev = self.tensors[0].device if n else torch.device("cuda", torch.cuda.current_device())
        self.device, self.index = dev, dev.index if dev.type == "cuda" else -1
        for t in self.tensors:
            if (not isinstance(t, torch.Tensor) or t.dtype not in DTYPES or t.get_device() != self.index or self.index < 0
                    or not t.is_contiguous()):
                raise b.DgnError(b.DGN_ERR_INVALID_ARG, "TensorList")
        self._numel = np.fromiter((t.numel() for t in self.tensors), np.int64, n)
        data = np.fromiter((t.data_ptr() for t in self.tensors), np.uint64, n)
        self._memory = [t.untyped_storage() for t in self.tensors]
        types = np.fromiter((DTYPES[t.dtype] for t in self.tensors), np.int32, n)
        desc = b.dgn_list_desc(count=n, data=data.ctypes.data, numel=self._numel.ctypes.data, dtype=types.ctypes.data)
        self.handle = None
        rc, nb = b.dgn_list_workspace(desc)
        b._check(rc, "dgn_list_workspace")
        self._mem = torch.empty(nb, dtype=torch.uint8, device=dev)
        rc, self.handle = b.dgn_list_build(desc, self._mem, nb, _queue(self.index, stream))
        b._check(rc, "dgn_list_build")

    def __len__(self):
        return len(self.tensors)

    def close(self, destroy=b._lib.dgn_list_destroy):      # (bound here: a list may outlive the module's names)
        if self.handle:
            destroy(self.handle)
            self.handle = None

    def __del__(self):
        if getattr(self, "handle", None):
            self.close()


def _reach(lst, num_sets, mask, ids):
    if mask is None:
        _need(ids is None, "tensor_ids without tensor_mask")
        return b.dgn_reach(num_sets)
    at = lst.index
    if mask.dtype is not torch.int64 or mask.dim() != 1 or mask.get_device() != at or not mask.is_contiguous():
        raise b.DgnError(b.DGN_ERR_INVALID_ARG, "tensor_mask")
    # (a mask of no words has no address, which would say that there is no mask: the list's own is not read)
    return b.dgn_reach(num_sets, mask.data_ptr() or lst._mem.data_ptr(), mask.numel(),
                       _dense(ids, (len(lst),), torch.int32, at, "tensor_ids"))


class GradientBuffers:
    """Norms of a list of gradients for up to 64 target sets, and clipping by them.

    ``mask``: int64 words as ``PruneBuffers.prune`` or ``backward_prune`` leave them in ``tensor_mask`` (bit q: target set
    q needs the tensor); ``ids``: int32, the graph's tensor that each entry of the list stands for.  Without ``mask``
    every set needs every tensor."""

    def __init__(self, grads: TensorList, num_sets: int = 1):
        self.grads, self.num_sets = grads, num_sets
        rc, sb = b.dgn_list_norms_workspace(grads.handle)
        b._check(rc, "dgn_list_norms_workspace")
        self.norms = torch.empty(max(num_sets, 1), dtype=torch.float32, device=grads.device)
        self._scratch, self._scratch_bytes = torch.empty(sb, dtype=torch.uint8, device=grads.device), sb

    def norm(self, mask=None, ids=None, stream=None):
        """Fills ``norms`` [num_sets]."""
        r = _reach(self.grads, self.num_sets, mask, ids)
        b._check(b._lib.dgn_list_norms(self.grads.handle, ctypes.byref(r), self.norms.data_ptr(), self._scratch.data_ptr(),
                                       self._scratch_bytes, _queue(self.grads.index, stream)), "dgn_list_norms")

    def clip(self, out: TensorList, max_norm, eps=1e-6, mask=None, ids=None, stream=None):
        """Writes the gradients, scaled so that no set's norm is above ``max_norm``, to ``out`` (may be the list itself);
        goes by ``norms`` as the last ``norm`` call left them."""
        at = self.grads.index
        if out.index != at:
            raise b.DgnError(b.DGN_ERR_INVALID_ARG, "clip: a list of another device")
        r = _reach(self.grads, self.num_sets, mask, ids)
        b._check(b._lib.dgn_list_clip(self.grads.handle, out.handle, ctypes.byref(r), self.norms.data_ptr(), max_norm, eps,
                                      _queue(at, stream)), "dgn_list_clip")


class AdamBuffers:
    """The lists of an Adam update: gradients, parameters and both moments (float32), where the new ones go (default: in
    place), and a list that receives the new parameters once more in its own types."""

    def __init__(self, grads: TensorList, params: TensorList, m: TensorList, v: TensorList, out_params=None, out_m=None,
                 out_v=None, copy=None):
        self._all = [t for t in (grads, params, m, v, out_params, out_m, out_v, copy) if t is not None]
        self._need_open()
        _need(all(t.index == grads.index for t in self._all), "AdamBuffers: lists of several devices")
        self.grads = grads
        self._lists = b.dgn_adam_lists(*(None if t is None else t.handle for t in (grads, params, m, v, out_params, out_m, out_v, copy)))

    def _need_open(self):       # (the library keeps nothing of a list that is closed, and takes none for `in place`)
        if None in [t.handle for t in self._all]:
            raise b.DgnError(b.DGN_ERR_INVALID_ARG, "AdamBuffers: a closed list")

    def step(self, lr, beta1, beta2, eps, weight_decay, step, norms=None, max_norm=1.0, clip_eps=1e-6, mask=None, ids=None,
             num_sets=None, skip_nonfinite=False, stream=None):
        """``norms`` (of ``GradientBuffers``): gradients are scaled as ``clip`` would; ``num_sets`` defaults to their number.
        Captured into a graph, every replay applies these rates and the bias corrections of this ``step``."""
        self._need_open()
        if norms is not None:
            num_sets = norms.numel() if num_sets is None else num_sets
            _need(norms.dtype is torch.float32 and norms.is_contiguous() and norms.numel() >= num_sets
                  and norms.get_device() == self.grads.index, "norms")
        r = _reach(self.grads, (64 if mask is not None else 1) if num_sets is None else num_sets, mask, ids)
        o = b.dgn_adam_options(lr, beta1, beta2, eps, weight_decay, step, int(skip_nonfinite), max_norm, clip_eps)
        b._check(b._lib.dgn_list_adam(ctypes.byref(self._lists), ctypes.byref(r), None if norms is None else norms.data_ptr(),
                                      ctypes.byref(o), _queue(self.grads.index, stream)), "dgn_list_adam")
