"""Timed cases of the operators of a selective recurrent layer: the short causal convolution and the selective scan
(forward, training step, one token), and dropout that is added to a residual.

``run`` computes them with elementary torch operations in 32 bits, or, where ``own`` is set, with the library's
entry points on the same inputs; ``exact`` gives the definition in 64 bits.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
MASK = 0xFFFFFFFF


def listed():
    return [
        # the convolution of one short prompt: everything is latency
        {"name": "conv_prompt", "op": "conv", "dtype": "bf16", "act": "silu", "taps": 4, "seqs": 1, "tokens": 257,
         "channels": 1000, "state": False},
        # a training step over a packed batch of sequences of very different lengths, some of them empty, that go on from
        # earlier ones
        {"name": "conv_train", "op": "conv_train", "dtype": "f16", "act": "silu", "taps": 4, "seqs": 96, "tokens": 65301,
         "channels": 1024, "state": True},
        # one token for each of 512 requests, a few of the batch's rows idle
        {"name": "conv_step", "op": "conv_step", "dtype": "bf16", "act": "silu", "taps": 4, "rows": 512, "slots": 700,
         "channels": 2048},
        # the scan of one short prompt
        {"name": "select_prompt", "op": "select", "dtype": "bf16", "seqs": 1, "tokens": 257, "channels": 512, "states": 16,
         "groups": 1, "z": True, "h0": False},
        # prompts of very different lengths, packed; some go on from earlier states
        {"name": "select_ragged", "op": "select", "dtype": "bf16", "seqs": 96, "tokens": 32771, "channels": 2048,
         "states": 16, "groups": 1, "z": True, "h0": True},
        # a training step of an ordinary layer
        {"name": "select_train", "op": "select_train", "dtype": "bf16", "seqs": 8, "tokens": 16384, "channels": 1024,
         "states": 16, "groups": 1, "z": True, "h0": False},
        # a training step in 32 bits on a narrow layer, two groups, an odd number of states, without the outer gate
        {"name": "select_train_f32", "op": "select_train", "dtype": "f32", "seqs": 5, "tokens": 5001, "channels": 400,
         "states": 9, "groups": 2, "z": False, "h0": True},
        # a training step on one long sequence with many states
        {"name": "select_train_long", "op": "select_train", "dtype": "f16", "seqs": 1, "tokens": 12001, "channels": 512,
         "states": 64, "groups": 4, "z": True, "h0": False},
        # one token for each of a few requests
        {"name": "select_step_few", "op": "select_step", "dtype": "bf16", "rows": 4, "slots": 64, "channels": 1000,
         "states": 16, "groups": 1, "z": True},
        # one token for each of 1,024 requests, states in a pool that is larger
        {"name": "select_step_many", "op": "select_step", "dtype": "bf16", "rows": 1024, "slots": 1200, "channels": 2048,
         "states": 16, "groups": 1, "z": True},
        # dropout of a few rows: launches
        {"name": "dropout_small", "op": "dropout", "dtype": "bf16", "rows": 16, "columns": 1000, "rate": 0.1},
        # dropout of a layer's outputs added to the residual, and its gradient
        {"name": "dropout_train", "op": "dropout", "dtype": "bf16", "rows": 65537, "columns": 1024, "rate": 0.1},
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["conv", "conv_train", "conv_step", "select", "select", "select_train", "select_train", "select_step",
                     "dropout"])
    case = {"op": op, "dtype": rng.choice(["f32", "bf16", "f16"])}
    if op == "dropout":
        columns = _log(rng, 33, 4096)
        return {**case, "rows": _log(rng, 3, 60_000_000 // columns), "columns": columns, "rate": rng.choice([0.0, 0.1, 0.35, 0.5])}
    if op.startswith("conv"):
        case.update(act=rng.choice(["silu", "silu", "none"]), taps=rng.choice([2, 3, 4, 4]), channels=_log(rng, 33, 2500))
        if op == "conv_step":
            rows = _log(rng, 1, 2048)
            return {**case, "rows": rows, "slots": rows + _log(rng, 1, 500)}
        tokens = _log(rng, 17, min(60_000_000 // case["channels"], 65_000))
        return {**case, "seqs": _log(rng, 1, min(300, tokens)), "tokens": tokens, "state": rng.random() < 0.5}
    states, groups = rng.choice([3, 8, 16, 16, 16, 32, 64, 128]), rng.choice([1, 1, 2, 4])
    channels = max(1, _log(rng, 32, 2048) // groups) * groups
    case.update(channels=channels, states=states, groups=groups, z=rng.random() < 0.7)
    if op == "select_step":
        rows = _log(rng, 1, max(2, min(1024, 33_000_000 // (channels * states))))
        return {**case, "rows": rows, "slots": rows + _log(rng, 1, 150)}
    most = 260_000_000 // (channels * states)
    tokens = _log(rng, 17, min(most, 20_000))
    return {**case, "seqs": _log(rng, 1, min(300, tokens)), "tokens": tokens, "h0": rng.random() < 0.5}


def _lengths(case, gen):
    """Lengths of the sequences: uneven, a seventh of them empty where there are enough, in all case["tokens"]."""
    n, total = case["seqs"], case["tokens"]
    if n == 1:
        return [total]
    share = torch.rand(n, generator=gen) ** 2 + 0.02
    share[torch.arange(n) % 7 == 3] = 0.0
    ends = torch.round(torch.cumsum(share, 0) / share.sum() * total).long().clamp(max=total)
    ends[-1] = total
    return torch.diff(ends, prepend=ends.new_zeros(1)).tolist()


def prepare(case, seed):
    st = _inputs(case, seed)
    if own:
        _owners(st)
    return st


def _inputs(case, seed):
    gen = torch.Generator().manual_seed(seed)
    dev = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, device="cuda", generator=dev)  # noqa: E731
    uniform = lambda *shape: torch.rand(*shape, device="cuda", generator=dev)  # noqa: E731
    st, dtype, op = {"case": case}, DTYPES[case["dtype"]], case["op"]
    if op == "dropout":
        shape = (case["rows"], case["columns"])
        st["x"], st["residual"], st["dy"] = (normal(*shape).to(dtype) for _ in range(3))
        # a seed of 64 bits, and the number of the step
        st["key"] = torch.randint(-2**62, 2**62, (2,), generator=gen).cuda()
        return st
    rows, c = case["rows" if "rows" in case else "tokens"], case["channels"]
    if "rows" in case:
        slots = torch.randperm(case["slots"], generator=gen)[:rows].to(torch.int32)
        if rows > 8:
            slots[::37] = -1                        # rows of the batch that no request has taken
        st["slots"] = slots.cuda()
    else:
        st["lens"] = torch.tensor(_lengths(case, gen))
        st["some"] = st["lens"].nonzero()[:, 0].cuda()
        rowptr = torch.tensor([0] + torch.cumsum(st["lens"], 0).tolist(), device="cuda")
        st["rowptr"] = rowptr
        # the sequence of each row, and its place in it
        st["seq"] = torch.repeat_interleave(torch.arange(case["seqs"], device="cuda"), st["lens"].cuda())
        st["pos"] = torch.arange(rows, device="cuda") - rowptr[st["seq"]]
    st["x"] = normal(rows, c).to(dtype)
    if op.startswith("conv"):
        k = case["taps"]
        st["weight"], st["bias"] = normal(c, k) / math.sqrt(k), normal(c) * 0.1
        if op == "conv_step":
            st["pool"] = normal(case["slots"], k - 1, c).to(dtype)
            st["next"] = torch.cat((st["pool"], st["pool"][:1]))        # and a row that nobody reads
            return st
        st["state0"] = normal(case["seqs"], k - 1, c).to(dtype) if case["state"] else None
        if op == "conv_train":
            st["dy"] = normal(rows, c).to(dtype)
            st["dfinal"] = normal(case["seqs"], k - 1, c).to(dtype) if case["state"] else None
        return st
    n, g = case["states"], case["groups"]
    # decays of 1, 2, 3 ... a unit of time; steps of a thousandth to a tenth, as layers of this kind begin their training
    st["A"] = -torch.arange(1, n + 1, device="cuda") * (1 + 0.1 * normal(c, n).clamp(-3, 3))
    step = torch.exp(uniform(c) * math.log(100.0) + math.log(1e-3))
    st["delta_bias"] = step + torch.log(-torch.expm1(-step))
    st["delta"] = (normal(rows, c) * 0.7).to(dtype)
    st["B"], st["C"] = normal(rows, g * n).to(dtype), normal(rows, g * n).to(dtype)
    st["D"] = 1 + 0.1 * normal(c)
    st["z"] = normal(rows, c).to(dtype) if case["z"] else None
    if op == "select_step":
        st["pool"] = normal(case["slots"], c, n)
        st["next"] = torch.cat((st["pool"], st["pool"][:1]))
        return st
    st["h0"] = normal(case["seqs"], c, n) if case["h0"] else None
    if op == "select_train":
        st["dy"] = normal(rows, c).to(dtype)
        st["dfinal"] = normal(case["seqs"], c, n) if case["h0"] else None
    return st


def _owners(st):
    """What a program makes once: owners of outputs and scratch."""
    import paper_1707_08265_amd as dgn
    case, op = st["case"], st["case"]["op"]
    dtype = DTYPES[case["dtype"]]
    if op == "dropout":
        st["buf"] = dgn.DropoutBuffers(case["rows"], case["columns"], case["rate"], dtype=dtype)
    elif op == "conv_step":
        st["buf"] = dgn.ConvStepBuffers(case["rows"], case["slots"], case["channels"], taps=case["taps"], activation=case["act"],
                                        dtype=dtype)
    elif op.startswith("conv"):
        st["buf"] = dgn.ConvBuffers(case["tokens"], case["seqs"], case["channels"], taps=case["taps"], activation=case["act"],
                                    dtype=dtype, train=op == "conv_train")
    elif op == "select_step":
        st["buf"] = dgn.SelectiveStepBuffers(case["rows"], case["slots"], case["channels"], num_states=case["states"],
                                             num_groups=case["groups"], dtype=dtype)
    else:
        st["buf"] = dgn.SelectiveBuffers(case["tokens"], case["seqs"], case["channels"], num_states=case["states"],
                                         num_groups=case["groups"], dtype=dtype, train=op == "select_train")


def run(state):
    return (_own if own else _plain)(state)


def _own(st):
    op, b = st["case"]["op"], st["buf"]
    if op == "dropout":
        b.forward(st["x"], st["key"], residual=st["residual"])
        b.backward(st["dy"], st["key"])
        return [b.y, b.dx]
    if op == "conv_step":
        b.step(st["x"], st["weight"], st["slots"], st["pool"], st["next"][:-1], bias=st["bias"])
        return [b.y, st["next"][:-1]]
    if op.startswith("conv"):
        b.forward(st["x"], st["weight"], st["rowptr"], bias=st["bias"], state0=st["state0"])
        if op == "conv":
            return [b.y, b.final]
        b.backward(st["x"], st["weight"], st["rowptr"], st["dy"], bias=st["bias"], state0=st["state0"], dfinal=st["dfinal"])
        return [b.y, b.final, b.dx, b.dweight, b.dbias, b.dstate0]
    more = {"D": st["D"], "delta_bias": st["delta_bias"], "z": st["z"]}
    if op == "select_step":
        b.step(st["x"], st["delta"], st["A"], st["B"], st["C"], st["slots"], st["pool"], st["next"][:-1], **more)
        return [b.y, st["next"][:-1]]
    b.forward(st["x"], st["delta"], st["A"], st["B"], st["C"], st["rowptr"], h0=st["h0"], **more)
    if op == "select":
        return [b.y, b.final]
    b.backward(st["x"], st["delta"], st["A"], st["B"], st["C"], st["rowptr"], st["dy"], h0=st["h0"], dfinal=st["dfinal"], **more)
    return [b.y, b.final, b.dx, b.ddelta, b.dA, b.dB, b.dC, b.dD, b.ddelta_bias, *([b.dz] if st["case"]["z"] else []), b.dh0]


def _plain(st):
    op = st["case"]["op"]
    if op == "dropout":
        return _plain_dropout(st)
    return {"conv": _plain_conv, "conv_step": _plain_conv_step, "conv_train": _plain_conv, "select": _plain_select,
            "select_step": _plain_select_step, "select_train": _plain_select}[op](st)


def _words(block, key):
    """Philox 4x32 with 10 rounds (Salmon et al., 2011) of the counters (block, offset), as four tensors of 32-bit numbers
    in 64; the key is (seed, offset)."""
    low = lambda v: v & MASK  # noqa: E731
    high = lambda v: (v >> 32) & MASK  # noqa: E731
    c0, c1 = low(block), high(block)
    c2, c3 = low(key[1]).expand_as(block), high(key[1]).expand_as(block)
    k0, k1 = low(key[0]), high(key[0])
    for _ in range(10):
        p, q = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = high(q) ^ c1 ^ k0, low(q), high(p) ^ c3 ^ k1, low(p)
        k0, k1 = low(k0 + 0x9E3779B9), low(k1 + 0xBB67AE85)
    return c0, c1, c2, c3


def _plain_dropout(st):
    case = st["case"]
    dtype, n = DTYPES[case["dtype"]], case["rows"] * case["columns"]
    drop = round(case["rate"] * 65536)
    words = _words(torch.arange(-(-n // 8), device="cuda"), st["key"])
    draws = torch.stack([part for w in words for part in (w & 0xFFFF, w >> 16)], 1).flatten()[:n]
    keep = (draws >= drop).view(case["rows"], -1)
    scale = 65536 / (65536 - drop)
    y = torch.where(keep, st["x"].float() * scale, 0.0) + st["residual"].float()
    return [y.to(dtype), torch.where(keep, st["dy"].float() * scale, 0.0).to(dtype)]


def _activate(case, p):
    return p * torch.sigmoid(p) if case["act"] == "silu" else p


def _back(st, s, x):
    """Row t - s of the sequence of each row t, in 32 bits: of the state where the sequence has none so early."""
    if s == 0:
        return x
    out = torch.zeros_like(x)
    out[s:] = x[:-s]
    early = (st["pos"] < s).nonzero()[:, 0]
    out[early] = 0.0
    if st["state0"] is not None:
        out[early] = st["state0"][st["seq"][early], st["case"]["taps"] - 1 + st["pos"][early] - s].float()
    return out


def _plain_conv(st):
    case, k, rows = st["case"], st["case"]["taps"], st["case"]["tokens"]
    dtype, w, x = DTYPES[case["dtype"]], st["weight"], st["x"].float()
    p = st["bias"].expand_as(x)
    for j in range(k):
        p = p + w[:, j] * _back(st, k - 1 - j, x)
    # the last k - 1 rows of each sequence: of its state where it has fewer
    at = st["lens"].cuda()[:, None] - (k - 1) + torch.arange(k - 1, device="cuda")
    inside = (at >= 0)[:, :, None]
    row = (st["rowptr"][:-1, None] + at).clamp(0, rows - 1)
    left = torch.zeros(case["seqs"], k - 1, case["channels"], device="cuda", dtype=dtype)
    if st["state0"] is not None:
        left = st["state0"][torch.arange(case["seqs"], device="cuda")[:, None], (k - 1 + at).clamp(max=k - 2)]
    out = [_activate(case, p).to(dtype), torch.where(inside, st["x"][row], left)]
    if case["op"] == "conv":
        return out
    g = st["dy"].float()
    if case["act"] == "silu":
        s = torch.sigmoid(p)
        g = g * s * (1 + p * (1 - s))
    dx, dstate = w[:, k - 1] * g, torch.zeros(left.shape, device="cuda")
    dw = torch.empty_like(w)
    dw[:, k - 1] = (g * x).sum(0)
    for s in range(1, k):
        tap = w[:, k - 1 - s]
        late = st["pos"] >= s
        dx[:-s] += torch.where(late[s:, None], tap * g[s:], 0.0)
        early = (~late).nonzero()[:, 0]
        dstate[st["seq"][early], k - 1 + st["pos"][early] - s] += tap * g[early]
        dw[:, k - 1 - s] = (g * _back(st, s, x)).sum(0)
    if st["dfinal"] is not None:
        q, i = inside[:, :, 0].nonzero(as_tuple=True)
        dx[row[q, i]] += st["dfinal"][q, i].float()
        q, i = (~inside[:, :, 0]).nonzero(as_tuple=True)
        dstate[q, k - 1 + at[q, i]] += st["dfinal"][q, i].float()
    return out + [dx.to(dtype), dw, g.sum(0), dstate.to(dtype)]


def _plain_conv_step(st):
    case, dtype = st["case"], DTYPES[st["case"]["dtype"]]
    live, slot = st["slots"] >= 0, st["slots"].long()
    window = torch.cat((st["pool"][slot.clamp(min=0)], st["x"][:, None]), 1)
    p = (window.float() * st["weight"].t()).sum(1) + st["bias"]
    st["next"][torch.where(live, slot, case["slots"])] = window[:, 1:]
    return [torch.where(live[:, None], _activate(case, p), 0.0).to(dtype), st["next"][:-1]]


def _linear_scan(a, u, longest):
    """h_t = a_t h_{t-1} + u_t down the rows by doubling; a is zero where a sequence begins."""
    shift = 1
    while shift < longest:
        u = torch.cat((u[:shift], u[shift:] + a[shift:] * u[:-shift]))
        a = torch.cat((a[:shift], a[shift:] * a[:-shift]))
        shift *= 2
    return u


def _by_channel(case, t):
    """[rows][groups * states] -> [rows][channels][states] in 32 bits."""
    t = t.float().view(-1, case["groups"], 1, case["states"])
    return t.expand(-1, -1, case["channels"] // case["groups"], -1).reshape(len(t), case["channels"], case["states"])


def _by_group(case, t):
    """The sum over each group's channels: [rows][channels][states] -> [rows][groups * states]."""
    return t.view(len(t), case["groups"], -1, case["states"]).sum(2).flatten(1)


def _steps(st):
    """softplus(delta + its bias)."""
    v = st["delta"].float() + st["delta_bias"]
    return v.clamp(min=0) + torch.log1p(torch.exp(-v.abs())), v


def _plain_select(st):
    case, dtype = st["case"], DTYPES[st["case"]["dtype"]]
    x, z = st["x"].float(), None if st["z"] is None else st["z"].float()
    d, v = _steps(st)
    a, b = torch.exp(d[:, :, None] * st["A"]), _by_channel(case, st["B"])
    some = st["some"]
    first, last = st["rowptr"][:-1][some], st["rowptr"][1:][some] - 1
    longest = int(st["lens"].max())
    h0 = torch.zeros(case["seqs"], *a.shape[1:], device="cuda") if st["h0"] is None else st["h0"]
    cut = a.clone()
    cut[first] = 0.0
    u = (d * x)[:, :, None] * b
    u[first] += a[first] * h0[some]
    h = _linear_scan(cut, u, longest)
    del u, cut
    final = h0.clone()
    final[some] = h[last]
    c = _by_channel(case, st["C"])
    y = (h * c).sum(2) + st["D"] * x
    out = [(y if z is None else y * z * torch.sigmoid(z)).to(dtype), final]
    if case["op"] == "select":
        return out
    o, dz = st["dy"].float(), None
    if z is not None:
        s = torch.sigmoid(z)
        dz = (o * y * s * (1 + z * (1 - s))).to(dtype)
        o = o * z * s
    dc = _by_group(case, o[:, :, None] * h)
    before = torch.cat((torch.zeros_like(h[:1]), h[:-1]))
    before[first] = h0[some]
    del h
    e = o[:, :, None] * c
    del c
    if st["dfinal"] is not None:
        e[last] += st["dfinal"][some]
    back = torch.cat((a[1:], torch.zeros_like(a[:1])))
    back[last] = 0.0
    e = _linear_scan(back.flip(0), e.flip(0), longest).flip(0)
    del back
    dh0 = torch.zeros_like(h0) if st["dfinal"] is None else st["dfinal"].clone()
    dh0[some] = a[first] * e[first]
    db = _by_group(case, e * (d * x)[:, :, None])
    eb = (e * b).sum(2)
    del b
    w = e * a * before
    da = (w * d[:, :, None]).sum(0)
    ddelta = ((w * st["A"]).sum(2) + eb * x) * torch.sigmoid(v)
    out += [(st["D"] * o + d * eb).to(dtype), ddelta.to(dtype), da, db.to(dtype), dc.to(dtype), (o * x).sum(0), ddelta.sum(0)]
    return out + ([] if dz is None else [dz]) + [dh0]


def _plain_select_step(st):
    case, dtype = st["case"], DTYPES[st["case"]["dtype"]]
    live, slot, x = st["slots"] >= 0, st["slots"].long(), st["x"].float()
    d, _ = _steps(st)
    h = torch.exp(d[:, :, None] * st["A"]) * st["pool"][slot.clamp(min=0)] + (d * x)[:, :, None] * _by_channel(case, st["B"])
    y = (h * _by_channel(case, st["C"])).sum(2) + st["D"] * x
    if st["z"] is not None:
        z = st["z"].float()
        y = y * z * torch.sigmoid(z)
    st["next"][torch.where(live, slot, case["slots"])] = h
    return [torch.where(live[:, None], y, 0.0).to(dtype), st["next"][:-1]]


def work(case):
    s, op = SIZE[case["dtype"]], case["op"]
    if op == "dropout":
        n = case["rows"] * case["columns"]
        return {"bytes": 5 * s * n + 16, "flops": 3 * n}
    c = case["channels"]
    busy = case["rows"] - (-(-case["rows"] // 37) if case["rows"] > 8 else 0) if "rows" in case else 0
    if op.startswith("conv"):
        k = case["taps"]
        each, weights = 2 * k + (4 if case["act"] == "silu" else 0), 4 * c * (k + 1)
        if op == "conv_step":
            return {"bytes": busy * c * s * (2 * k - 1) + case["rows"] * (c * s + 4) + weights, "flops": busy * c * each}
        n, state = case["tokens"], case["seqs"] * (k - 1) * c * s
        forward = 2 * n * c * s + weights + state * (2 if case["state"] else 1)
        if op == "conv":
            return {"bytes": forward, "flops": n * c * each}
        return {"bytes": forward + 3 * n * c * s + 2 * weights + state * (3 if case["state"] else 1), "flops": n * c * (2 * each + 4 * k + 6)}
    n, g, z = case["states"], case["groups"], 1 if case["z"] else 0
    each, params = c * (7 * n + 10), 4 * c * (n + 2)
    row = s * ((2 + z) * c + 2 * g * n)
    if op == "select_step":
        return {"bytes": busy * (row + 8 * c * n) + case["rows"] * (c * s + 4) + params, "flops": busy * each}
    t, state = case["tokens"], 4 * case["seqs"] * c * n
    forward = t * (row + c * s) + params + state * (2 if case["h0"] else 1)
    if op == "select":
        return {"bytes": forward, "flops": t * each}
    return {"bytes": forward + t * (2 * row + c * s) + 2 * params + state * (3 if case["h0"] else 1),
            "flops": t * (each + c * (21 * n + 30))}


def exact(case, seed):
    st = _inputs(case, seed)
    op = case["op"]
    if op == "dropout":
        return _exact_dropout(st)
    return _exact_conv(st) if op.startswith("conv") else _exact_select(st)


def _exact_dropout(st):
    n = st["x"].numel()
    key = [int(v) % 2**64 for v in st["key"].tolist()]
    block = np.arange(-(-n // 8), dtype=np.uint64)
    low, shift = np.uint64(MASK), np.uint64(32)
    ctr = [block & low, block >> shift, np.uint64(key[1] & MASK), np.uint64(key[1] >> 32)]
    for r in range(10):
        first, second = ctr[0] * np.uint64(0xD2511F53), ctr[2] * np.uint64(0xCD9E8D57)
        ks = [np.uint64(((key[0] & MASK) + r * 0x9E3779B9) & MASK), np.uint64(((key[0] >> 32) + r * 0xBB67AE85) & MASK)]
        ctr = [(second >> shift) ^ ctr[1] ^ ks[0], second & low, (first >> shift) ^ ctr[3] ^ ks[1], first & low]
    draws = np.empty((len(block), 8), dtype=np.uint16)
    for i, word in enumerate(ctr):
        draws[:, 2 * i], draws[:, 2 * i + 1] = word & np.uint64(65535), word >> np.uint64(16)
    dropped = int(np.floor(st["case"]["rate"] * 65536 + 0.5))
    mask = torch.from_numpy((draws.reshape(-1)[:n] >= dropped).reshape(tuple(st["x"].shape))).cuda()
    factor = mask.double() / (1 - dropped / 65536)
    return [st["residual"].double() + st["x"].double() * factor, st["dy"].double() * factor]


def _exact_conv(st):
    case, k = st["case"], st["case"]["taps"]
    silu, w, bias = case["act"] == "silu", st["weight"].double(), st["bias"].double()
    value = lambda p: p / (1 + torch.exp(-p)) if silu else p  # noqa: E731
    if case["op"] == "conv_step":
        y, pool = torch.zeros(st["x"].shape, dtype=torch.float64, device="cuda"), st["pool"].double()
        for r, slot in enumerate(st["slots"].tolist()):
            if slot >= 0:
                seen = torch.cat((pool[slot], st["x"][r:r + 1].double()))
                y[r] = value(bias + (seen * w.t()).sum(0))
                pool[slot] = seen[1:]
        return [y, pool]
    # sequence by sequence, with the rows before it in front
    parts = [[] for _ in range(4)]
    dw, dbias = torch.zeros_like(w), torch.zeros_like(bias)
    start = 0
    for q, n in enumerate(st["lens"].tolist()):
        rows = slice(start, start + n)
        start += n
        early = torch.zeros(k - 1, case["channels"], dtype=torch.float64, device="cuda") if st["state0"] is None else st["state0"][q].double()
        seen = torch.cat((early, st["x"][rows].double()))
        p = bias + sum(seen[j:j + n] * w[:, j] for j in range(k))
        parts[0].append(value(p))
        parts[1].append(seen[n:])
        if case["op"] == "conv":
            continue
        g = st["dy"][rows].double()
        if silu:
            s = 1 / (1 + torch.exp(-p))
            g = g * (s + p * s * (1 - s))
        grad = torch.zeros_like(seen)
        for j in range(k):
            grad[j:j + n] += g * w[:, j]
            dw[:, j] += (g * seen[j:j + n]).sum(0)
        dbias += g.sum(0)
        if st["dfinal"] is not None:
            grad[n:] += st["dfinal"][q].double()
        parts[2].append(grad[k - 1:])
        parts[3].append(grad[:k - 1])
    y, final = torch.cat(parts[0]), torch.stack(parts[1])
    return [y, final] if case["op"] == "conv" else [y, final, torch.cat(parts[2]), dw, dbias, torch.stack(parts[3])]


def _exact_select(st):
    case, f = st["case"], torch.float64
    c, n, g = case["channels"], case["states"], case["groups"]
    x, A, D = st["x"].to(f), st["A"].to(f), st["D"].to(f)
    raw = st["delta"].to(f) + st["delta_bias"].to(f)
    d = torch.logaddexp(raw, torch.zeros_like(raw))
    group = torch.arange(c, device="cuda") // (c // g)
    B, C = (st[name].to(f).view(-1, g, n) for name in "BC")
    z = None if st["z"] is None else st["z"].to(f)
    gate = 1.0 if z is None else z / (1 + torch.exp(-z))
    if case["op"] == "select_step":
        y, pool = torch.zeros_like(x), st["pool"].to(f)
        for r, slot in enumerate(st["slots"].tolist()):
            if slot >= 0:
                pool[slot] = torch.exp(d[r][:, None] * A) * pool[slot] + (d[r] * x[r])[:, None] * B[r][group]
                y[r] = (pool[slot] * C[r][group]).sum(1) + D * x[r]
        return [y * gate, pool]
    start = st["rowptr"][:-1].tolist()
    order = sorted(range(case["seqs"]), key=lambda q: -int(st["lens"][q]))
    size = sorted((int(v) for v in st["lens"]), reverse=True)
    rows, seqs = torch.tensor([start[q] for q in order], device="cuda"), torch.tensor(order, device="cuda")
    h = torch.zeros(case["seqs"], c, n, dtype=f, device="cuda") if st["h0"] is None else st["h0"].to(f)[seqs]
    train = case["op"] == "select_train"
    y, before = torch.empty_like(x), torch.empty(len(x), c, n, dtype=f, device="cuda") if train else None
    active, live = [], case["seqs"]
    for t in range(size[0]):                        # token t of every sequence that has one
        while size[live - 1] <= t:
            live -= 1
        active.append(live)
        at = rows[:live] + t
        if train:
            before[at] = h[:live]
        h[:live] = torch.exp(d[at][:, :, None] * A) * h[:live] + (d[at] * x[at])[:, :, None] * B[at][:, group]
        y[at] = (h[:live] * C[at][:, group]).sum(2) + D * x[at]
    final = torch.empty_like(h)
    final[seqs] = h
    if not train:
        return [y * gate, final]
    o = st["dy"].to(f)
    dz = None
    if z is not None:
        s = 1 / (1 + torch.exp(-z))
        dz, o = o * y * (s + gate * (1 - s)), o * gate
    e = torch.zeros_like(h) if st["dfinal"] is None else st["dfinal"].to(f)[seqs]
    dx, dd, dA = torch.empty_like(x), torch.empty_like(x), torch.zeros_like(A)
    dB, dC = torch.empty(len(x), g * n, dtype=f, device="cuda"), torch.empty(len(x), g * n, dtype=f, device="cuda")
    total = lambda t: t.view(len(t), g, c // g, n).sum(2).flatten(1)  # noqa: E731
    for t in reversed(range(size[0])):
        live = active[t]
        at = rows[:live] + t
        step, put, b = d[at][:, :, None], x[at][:, :, None], B[at][:, group]
        a, early = torch.exp(step * A), before[at]
        full = e[:live] + o[at][:, :, None] * C[at][:, group]           # gradient of h_t
        dC[at] = total(o[at][:, :, None] * (a * early + step * put * b))
        dB[at] = total(full * step * put)
        inner = full * a * early
        dA += (inner * step).sum(0)
        dd[at] = (inner * A + full * b * put).sum(2)
        dx[at] = (full * b * step).sum(2) + D * o[at]
        e[:live] = a * full
    dh0 = torch.empty_like(e)
    dh0[seqs] = e
    ddelta = dd / (1 + torch.exp(-raw))
    out = [y * gate, final, dx, ddelta, dA, dB, dC, (o * x).sum(0), ddelta.sum(0)]
    return out + ([] if dz is None else [dz]) + [dh0]
