"""Timed cases of the operators on the values of a graph's tensors: the gated linear recurrence (forward, training
step, one token), the global gradient norm with clipping, and the update that applies it.

``run`` computes them with elementary torch operations in 32 bits, or, where ``own`` is set, with the library's
entry points on the same inputs; ``exact`` gives the definition in 64 bits.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
MAX_NORM, CLIP_EPS = 1.0, 1e-6
ADAM = {"lr": 3e-4, "beta1": 0.9, "beta2": 0.95, "eps": 1e-8, "weight_decay": 0.1, "step": 10}


def listed():
    return [
        # one short prompt: everything is latency
        {"name": "scan_prompt", "op": "scan", "kind": "sigmoid", "dtype": "bf16", "seqs": 1, "tokens": 257,
         "heads": 512, "group": 1, "h0": False},
        # the unrolled recurrence of 10,000 steps by 1,000 operators, as one operator: a single sequence, so all the
        # parallel work beyond 1,000 channels has to come from the length
        {"name": "scan_unrolled", "op": "scan", "kind": "sigmoid", "dtype": "bf16", "seqs": 1, "tokens": 10000,
         "heads": 1000, "group": 1, "h0": True},
        # a packed batch of requests of very different lengths, some of them empty
        {"name": "scan_ragged", "op": "scan", "kind": "decay", "dtype": "f16", "seqs": 96, "tokens": 65301,
         "heads": 2048, "group": 1, "h0": True},
        # a training step whose heads of 128 channels share a gate
        {"name": "train_heads", "op": "train", "kind": "decay", "dtype": "bf16", "seqs": 8, "tokens": 16384,
         "heads": 16, "group": 128, "h0": False},
        # a training step in 32 bits on a narrow layer
        {"name": "train_f32", "op": "train", "kind": "sigmoid", "dtype": "f32", "seqs": 5, "tokens": 20000,
         "heads": 400, "group": 1, "h0": True},
        # a training step on one very long sequence, a token past a power of two
        {"name": "train_long", "op": "train", "kind": "sigmoid", "dtype": "bf16", "seqs": 1, "tokens": 65537,
         "heads": 1024, "group": 1, "h0": False},
        # one token for each of a few requests
        {"name": "step_few", "op": "step", "kind": "sigmoid", "dtype": "bf16", "rows": 4, "slots": 64,
         "heads": 1000, "group": 1},
        # one token for each of 4,096 requests, states in a pool that is larger
        {"name": "step_many", "op": "step", "kind": "decay", "dtype": "bf16", "rows": 4096, "slots": 5000,
         "heads": 32, "group": 64},
        # the tensors of one small layer: launches
        {"name": "clip_layer", "op": "clip", "dtype": "f32", "layers": 2, "width": 64, "sets": 1},
        # 500 layers of width 400 in 16 and 32 bits, and 64 target sets that each reach some of them
        {"name": "clip_sets", "op": "clip", "dtype": "mixed", "layers": 500, "width": 400, "sets": 64},
        # the same small layer, updated
        {"name": "update_layer", "op": "update", "dtype": "f32", "layers": 2, "width": 64, "sets": 1},
        # 500 layers of width 400, gradients in 16 bits, parameters and moments in 32, a 16-bit copy of the parameters
        {"name": "update_wide", "op": "update", "dtype": "bf16", "layers": 500, "width": 400, "sets": 1},
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["scan", "scan", "train", "train", "step", "clip", "update"])
    if op in ("clip", "update"):
        layers = _log(rng, 1, 500)
        return {"op": op, "dtype": rng.choice(["f32", "bf16", "f16", "mixed"]), "layers": layers,
                "width": _log(rng, 24, min(1024, int(380 * math.sqrt(500 / layers)))), "sets": rng.choice([1, 1, 3, 64])}
    group = rng.choice([1, 1, 1, 8, 64, 96, 128, 200])
    heads = max(1, _log(rng, 32, 2500) // group)
    case = {"op": op, "kind": rng.choice(["sigmoid", "decay"]), "dtype": rng.choice(["f32", "bf16", "f16"]),
            "heads": heads, "group": group}
    if op == "step":
        rows = _log(rng, 1, 4096)
        return {**case, "rows": rows, "slots": rows + _log(rng, 1, 1000)}
    most = 30_000_000 // (heads * group)
    tokens = _log(rng, 17, min(most, 100_000))
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


def _shapes(case):
    """Tensors of the list: per layer a matrix, one of an odd shape, a bias and a single number."""
    w = case["width"]
    return [s for _ in range(case["layers"]) for s in (w * w, (w // 2) * (w + 1) + 1, w, 1)]


def _types(case):
    """Type of each tensor of the list: "mixed" has the matrices in 16 bits and what is small in 32."""
    if case["dtype"] != "mixed":
        return [case["dtype"]] * (4 * case["layers"])
    return ["bf16", "bf16", "f32", "f32"] * case["layers"]


def _views(flat, sizes):
    return list(torch.split(flat, sizes))


def _in_order(st, stores):
    """The tensors of the list, out of the store of each type."""
    place = [None] * len(st["sizes"])
    for t in st["names"]:
        for i, part in zip(st["entry"][t], _views(stores[t], st["part"][t])):
            place[i] = part
    return place


def prepare(case, seed):
    st = _inputs(case, seed)
    if own:
        _handles(st)
    return st


def _inputs(case, seed):
    gen = torch.Generator().manual_seed(seed)
    dev = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, device="cuda", generator=dev)  # noqa: E731
    st = {"case": case}
    if case["op"] in ("clip", "update"):
        sizes, types = _shapes(case), _types(case)
        st["sizes"], st["every"] = sizes, torch.tensor(sizes, device="cuda")
        st["names"] = sorted(set(types))
        # one store for each type, the tensors one after the other in it
        st["entry"] = {t: [i for i, u in enumerate(types) if u == t] for t in st["names"]}
        st["part"] = {t: [sizes[i] for i in st["entry"][t]] for t in st["names"]}
        st["at"] = {t: torch.tensor(st["entry"][t], device="cuda") for t in st["names"]}
        st["long"] = {t: torch.tensor(st["part"][t], device="cuda") for t in st["names"]}
        st["grad"] = {t: (normal(sum(st["part"][t])) * 0.01).to(DTYPES[t]) for t in st["names"]}
        # bit q of word i: target set q reaches tensor i; some tensors are reached by none
        bits = torch.ones(len(sizes), dtype=torch.int64)
        if case["sets"] > 1:
            reach = torch.rand(len(sizes), case["sets"], generator=gen) < 0.05
            bits = (reach.long() << torch.arange(case["sets"])).sum(1)
        st["bits"] = bits.cuda()
        if case["op"] == "update":
            total = sum(sizes)
            st["p"], st["m"] = normal(total) * 0.02, normal(total) * 0.001
            st["v"] = (normal(total) * 0.001).square()
            st["out"] = {k: torch.empty(total, device="cuda") for k in "pmv"}
            st["copy"] = torch.empty(total, device="cuda", dtype=torch.bfloat16)
        else:
            st["scaled"] = {t: torch.empty_like(g) for t, g in st["grad"].items()}
        return st
    dtype, heads, group = DTYPES[case["dtype"]], case["heads"], case["group"]
    rows = case["rows"] if case["op"] == "step" else case["tokens"]
    gate = normal(rows, heads) * 1.5 + 3.0
    st["gate"] = (gate if case["kind"] == "sigmoid" else torch.sigmoid(gate)).to(dtype)
    st["x"] = normal(rows, heads * group).to(dtype)
    if case["op"] == "step":
        slots = torch.randperm(case["slots"], generator=gen)[:rows].to(torch.int32)
        if rows > 8:
            slots[::37] = -1                        # rows of the batch that no request has taken
        st["slots"] = slots.cuda()
        st["pool"] = normal(case["slots"], heads * group)
        st["next"] = torch.cat((st["pool"], st["pool"][:1]))    # and a row that nobody reads
    else:
        lens = _lengths(case, gen)
        st["lens"] = torch.tensor(lens)
        st["some"] = st["lens"].nonzero()[:, 0].cuda()
        st["rowptr"] = torch.tensor([0] + torch.cumsum(st["lens"], 0).tolist(), device="cuda")
        st["h0"] = normal(case["seqs"], heads * group) if case["h0"] else None
        if case["op"] == "train":
            st["dy"] = normal(rows, heads * group).to(dtype)
            st["dfinal"] = normal(case["seqs"], heads * group) if case["h0"] else None
    return st


def _handles(st):
    """What a program makes once of its buffers: lists of tensors, and owners of outputs and scratch."""
    import paper_1707_08265_amd as dgn
    case = st["case"]
    if case["op"] in ("clip", "update"):
        grads = dgn.TensorList(_in_order(st, st["grad"]))
        st["norms"] = dgn.GradientBuffers(grads, case["sets"])
        if case["op"] == "clip":
            st["to"] = dgn.TensorList(_in_order(st, st["scaled"]))
            return
        stores = (st["p"], st["m"], st["v"], *(st["out"][k] for k in "pmv"), st["copy"])
        p, m, v, out_p, out_m, out_v, copy = (dgn.TensorList(_views(f, st["sizes"])) for f in stores)
        st["adam"] = dgn.AdamBuffers(grads, p, m, v, out_params=out_p, out_m=out_m, out_v=out_v, copy=copy)
        return
    channels, dtype = case["heads"] * case["group"], DTYPES[case["dtype"]]
    same = {"gate_group": case["group"], "kind": case["kind"], "dtype": dtype}
    if case["op"] == "step":
        st["buf"] = dgn.ScanStepBuffers(case["rows"], case["slots"], channels, **same)
    else:
        st["buf"] = dgn.ScanBuffers(case["tokens"], case["seqs"], channels, train=case["op"] == "train", **same)


def run(state):
    return (_own if own else _plain)(state)


def _own(st):
    op = st["case"]["op"]
    if op == "scan":
        b = st["buf"]
        b.forward(st["x"], st["gate"], st["rowptr"], h0=st["h0"])
        return [b.y, b.final]
    if op == "train":
        b = st["buf"]
        b.forward(st["x"], st["gate"], st["rowptr"], h0=st["h0"])
        b.backward(st["x"], st["gate"], st["rowptr"], st["dy"], h0=st["h0"], dfinal=st["dfinal"])
        return [b.y, b.final, b.dx, b.dgate, b.dh0]
    if op == "step":
        st["buf"].step(st["x"], st["gate"], st["slots"], st["pool"], st["next"][:-1])
        return [st["buf"].y, st["next"][:-1]]
    b = st["norms"]
    b.norm(st["bits"])
    if op == "clip":
        b.clip(st["to"], MAX_NORM, eps=CLIP_EPS, mask=st["bits"])
        return [b.norms, st["scaled"]]
    st["adam"].step(**ADAM, norms=b.norms, max_norm=MAX_NORM, clip_eps=CLIP_EPS, mask=st["bits"])
    return [b.norms, st["out"], st["copy"]]


def _linear_scan(a, u, longest):
    """h_t = a_t h_{t-1} + u_t down the rows by doubling; a is zero where a sequence begins."""
    shift = 1
    while shift < longest:
        u = torch.cat((u[:shift], u[shift:] + a[shift:] * u[:-shift]))
        a = torch.cat((a[:shift], a[shift:] * a[:-shift]))
        shift *= 2
    return u


def _gates(st, gate, x):
    """(a, 1 - a or None, x) in 32 bits, a gate for each channel."""
    wide = gate.float().repeat_interleave(st["case"]["group"], 1) if st["case"]["group"] > 1 else gate.float()
    if st["case"]["kind"] == "decay":
        return wide, None, x.float()
    return torch.sigmoid(wide), torch.sigmoid(-wide), x.float()


def _plain(st):
    case = st["case"]
    if case["op"] in ("clip", "update"):
        return _plain_list(st)
    dtype = DTYPES[case["dtype"]]
    a, b, x = _gates(st, st["gate"], st["x"])
    u = x if b is None else b * x
    if case["op"] == "step":
        live = st["slots"] >= 0
        h = a * st["pool"][st["slots"].long().clamp(min=0)] + u
        st["next"][torch.where(live, st["slots"].long(), case["slots"])] = h
        return [torch.where(live[:, None], h, 0.0).to(dtype), st["next"][:-1]]
    some = st["some"]
    first, last = st["rowptr"][:-1][some], st["rowptr"][1:][some] - 1
    longest = int(st["lens"].max())
    h0 = torch.zeros(case["seqs"], u.shape[1], device="cuda") if st["h0"] is None else st["h0"]
    cut = a.clone()
    cut[first] = 0.0
    u = u.clone()
    u[first] += a[first] * h0[some]
    h = _linear_scan(cut, u, longest)
    final = h0.clone()
    final[some] = h[last]
    if case["op"] == "scan":
        return [h.to(dtype), final]
    before = torch.cat((torch.zeros_like(h[:1]), h[:-1]))
    before[first] = h0[some]
    back = torch.cat((a[1:], torch.zeros_like(a[:1])))
    back[last] = 0.0
    e = st["dy"].float()
    if st["dfinal"] is not None:
        e = e.clone()
        e[last] += st["dfinal"][some]
    e = _linear_scan(back.flip(0), e.flip(0), longest).flip(0)
    dh0 = torch.zeros_like(h0) if st["dfinal"] is None else st["dfinal"].clone()
    dh0[some] = a[first] * e[first]
    if b is None:
        dx, dgate = e, e * before
    else:
        dx, dgate = b * e, a * b * e * (before - x)
    dgate = dgate.view(-1, case["heads"], case["group"]).sum(2)
    return [h.to(dtype), final, dx.to(dtype), dgate.to(dtype), dh0]


def _reach(st):
    return ((st["bits"][:, None] >> torch.arange(st["case"]["sets"], device="cuda")) & 1).bool()


def _plain_list(st):
    case = st["case"]
    sums = torch.zeros(len(st["sizes"]), device="cuda")
    for t in st["names"]:
        sums[st["at"][t]] = torch.segment_reduce(st["grad"][t].float().square(), "sum", lengths=st["long"][t], unsafe=True)
    reach = _reach(st)
    norms = (sums[:, None] * reach).sum(0).sqrt()
    factor = (MAX_NORM / (norms + CLIP_EPS)).clamp(max=1.0)
    factor = torch.where(reach, factor, 1.0).amin(1)
    scaled = {t: g.float() * factor[st["at"][t]].repeat_interleave(st["long"][t], output_size=g.numel())
              for t, g in st["grad"].items()}
    if case["op"] == "clip":
        return [norms, {t: g.to(DTYPES[t]) for t, g in scaled.items()}]
    # (of two types: a layer's tensors are its matrices in 16 bits, then the rest in 32)
    g = torch.cat([scaled[t].view(case["layers"], -1) for t in st["names"]], 1).flatten()
    k = ADAM
    m = k["beta1"] * st["m"] + (1 - k["beta1"]) * g
    v = k["beta2"] * st["v"] + (1 - k["beta2"]) * g.square()
    step = k["lr"] / (1 - k["beta1"] ** k["step"]) * m / ((v / (1 - k["beta2"] ** k["step"])).sqrt() + k["eps"])
    p = st["p"] * (1 - k["lr"] * k["weight_decay"]) - step
    if case["sets"] > 1:
        live = reach.any(1).repeat_interleave(st["every"], output_size=p.numel())
        p, m, v = torch.where(live, p, st["p"]), torch.where(live, m, st["m"]), torch.where(live, v, st["v"])
    return [norms, {"m": m, "p": p, "v": v}, p.to(torch.bfloat16)]


def work(case):
    size = {"f32": 4, "f16": 2, "bf16": 2}
    if case["op"] in ("clip", "update"):
        pairs = list(zip(_shapes(case), _types(case)))
        n, grads = sum(s for s, _ in pairs), sum(s * size[t] for s, t in pairs)
        if case["op"] == "clip":
            return {"bytes": 2 * grads + 8 * len(pairs), "flops": 3 * n}
        return {"bytes": grads + 26 * n + 8 * len(pairs), "flops": 16 * n}
    s, c = size[case["dtype"]], case["heads"] * case["group"]
    if case["op"] == "step":
        busy = case["rows"] - (-(-case["rows"] // 37) if case["rows"] > 8 else 0)
        return {"bytes": busy * (c * (s + 8) + case["heads"] * s) + case["rows"] * (c * s + 4), "flops": 4 * busy * c}
    n, state = case["tokens"], 4 * case["seqs"] * c
    forward = n * s * (2 * c + case["heads"]) + state * (2 if case["h0"] else 1)
    if case["op"] == "scan":
        return {"bytes": forward, "flops": 4 * n * c}
    return {"bytes": forward + n * s * (3 * c + 2 * case["heads"]) + state * (3 if case["h0"] else 1), "flops": 14 * n * c}


def exact(case, seed):
    st = _inputs(case, seed)
    if case["op"] in ("clip", "update"):
        return _exact_list(st)
    d, group = torch.float64, case["group"]
    gate, x = st["gate"].to(d), st["x"].to(d)
    heads = case["heads"]
    sigmoid = case["kind"] == "sigmoid"
    a = 1 / (1 + torch.exp(-gate)) if sigmoid else gate
    keep = 1 / (1 + torch.exp(gate)) if sigmoid else torch.ones_like(gate)
    x = x.view(-1, heads, group)
    a, keep = a[:, :, None], keep[:, :, None]
    if case["op"] == "step":
        y, pool = torch.zeros_like(x), st["pool"].to(d).view(-1, heads, group)
        for r, slot in enumerate(st["slots"].tolist()):
            if slot >= 0:
                pool[slot] = y[r] = a[r] * pool[slot] + keep[r] * x[r]
        return [y.flatten(1), pool.flatten(1)]
    start = st["rowptr"][:-1].tolist()
    order = sorted(range(case["seqs"]), key=lambda q: -int(st["lens"][q]))
    size = sorted((int(v) for v in st["lens"]), reverse=True)
    rows = torch.tensor([start[q] for q in order], device="cuda")
    seqs = torch.tensor(order, device="cuda")
    h = torch.zeros(case["seqs"], heads, group, dtype=d, device="cuda")
    if st["h0"] is not None:
        h = st["h0"].to(d).view(-1, heads, group)[seqs].clone()
    y, before = torch.empty_like(x), torch.empty_like(x)
    active, live = [], case["seqs"]
    for t in range(size[0]):                        # token t of every sequence that has one
        while size[live - 1] <= t:
            live -= 1
        active.append(live)
        at = rows[:live] + t
        before[at] = h[:live]
        h[:live] = a[at] * h[:live] + keep[at] * x[at]
        y[at] = h[:live]
    final = torch.empty_like(h)
    final[seqs] = h
    out = [y.flatten(1), final.flatten(1)]
    if case["op"] == "scan":
        return out
    dy = st["dy"].to(d).view(-1, heads, group)
    e = torch.zeros_like(h) if st["dfinal"] is None else st["dfinal"].to(d).view(-1, heads, group)[seqs].clone()
    dx, dgate = torch.empty_like(x), torch.empty_like(gate)
    for t in reversed(range(size[0])):
        live = active[t]
        at = rows[:live] + t
        full = e[:live] + dy[at]                    # gradient of h_t
        dx[at] = keep[at] * full
        if sigmoid:
            dgate[at] = (full * (before[at] - x[at])).sum(2) * (a[at] * keep[at])[:, :, 0]
        else:
            dgate[at] = (full * before[at]).sum(2)
        e[:live] = a[at] * full
    dh0 = torch.empty_like(e)
    dh0[seqs] = e
    return out + [dx.flatten(1), dgate, dh0.flatten(1)]


def _exact_list(st):
    case, d = st["case"], torch.float64
    grads = [g.to(d) for g in _in_order(st, st["grad"])]
    words = st["bits"].tolist()
    sums = torch.stack([(g * g).sum() for g in grads]).tolist()
    norms = [math.sqrt(math.fsum(v for v, w in zip(sums, words) if w >> q & 1)) for q in range(case["sets"])]
    least = [min([1.0] + [MAX_NORM / (norms[q] + CLIP_EPS) for q in range(case["sets"]) if w >> q & 1]) for w in words]
    scaled = [g * f for g, f in zip(grads, least)]
    norms = torch.tensor(norms, dtype=d)
    if case["op"] == "clip":
        return [norms, {t: torch.cat([scaled[i] for i in st["entry"][t]]) for t in st["names"]}]
    k, out = ADAM, {"p": [], "m": [], "v": []}
    for g, w, p, m, v in zip(scaled, words, *(_views(st[n].to(d), st["sizes"]) for n in "pmv")):
        if w:
            m = k["beta1"] * m + (1 - k["beta1"]) * g
            v = k["beta2"] * v + (1 - k["beta2"]) * g * g
            ahead = m / (1 - k["beta1"] ** k["step"])
            spread = torch.sqrt(v / (1 - k["beta2"] ** k["step"]))
            p = p - k["lr"] * (ahead / (spread + k["eps"]) + k["weight_decay"] * p)
        for name, value in zip("pmv", (p, m, v)):
            out[name].append(value)
    out = {n: torch.cat(parts) for n, parts in out.items()}
    return [norms, out, out["p"]]
