"""Plain 64-bit forms of the operators on tensor values, and how far a 32-bit computation may be off.

A bound is carried along with the values: S is the sum of the absolute values of all terms of a value, E the error.  A step
h' = a h + u forms each of its terms with a fixed number of 32-bit roundings whatever the order of the scan, so the error
obeys E' = a E + c S' with c that number of roundings; c also holds the error of the gate (exp to a few units times its
argument, one addition, one division).  Results are then rounded once to their type.
"""
import torch

U32 = 2.0 ** -24
ROUND = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
LEAST = {torch.float32: 2.0 ** -126, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -126}


def within(got, want, error, what):
    """|got - want| <= error + one rounding to got's type, element by element; what is no number has to be the same."""
    dtype, got = got.dtype, got.detach().double().cpu()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    room = error + ROUND[dtype] * (want.abs() + error) + LEAST[dtype]
    bad = ~((got - want).abs() <= room) & ~(got.isnan() & want.isnan()) & ~(got == want)
    assert not bad.any(), (what, int(bad.sum()), bad.nonzero()[:3].tolist(), got[bad][:3], want[bad][:3], room[bad][:3])


def gates(gate, kind, group):
    """(a, 1 - a or 1, roundings of a) for each channel, in 64 bits."""
    g = gate.double().cpu().repeat_interleave(group, 1)
    if kind == "decay":
        return g, torch.ones_like(g), torch.full_like(g, 4 * U32)
    return torch.sigmoid(g), torch.sigmoid(-g), (16 + 2 * g.abs().clamp(max=200)) * U32


def scan(x, gate, rowptr, kind, group, h0=None, dy=None, dfinal=None):
    """{name: (value, error)} of y and final, and of dx, dgate and dh0 if dy is given."""
    x, n, c = x.double().cpu(), x.shape[0], x.shape[1]
    a, b, slack = gates(gate, kind, group)
    bounds = rowptr.tolist()
    seqs = len(bounds) - 1
    zero = torch.zeros(seqs, c, dtype=torch.float64)
    h0 = zero if h0 is None else h0.double().cpu()
    y, size, err, before, bsize, berr = (torch.zeros(n, c, dtype=torch.float64) for _ in range(6))
    final, ferr = h0.clone(), zero.clone()
    for q in range(seqs):
        h, s, e = h0[q], h0[q].abs(), torch.zeros(c, dtype=torch.float64)
        for t in range(bounds[q], bounds[q + 1]):
            before[t], bsize[t], berr[t] = h, s, e
            h = a[t] * h + b[t] * x[t]
            s = a[t].abs() * s + b[t] * x[t].abs()
            e = a[t].abs() * e + slack[t] * s
            y[t], size[t], err[t] = h, s, e
        final[q], ferr[q] = h, e
    out = {"y": (y, err), "final": (final, ferr)}
    if dy is None:
        return out
    dy = dy.double().cpu()
    dfinal = zero if dfinal is None else dfinal.double().cpu()
    dx, dxerr, dg, dgsize, dgerr = (torch.zeros(n, c, dtype=torch.float64) for _ in range(5))
    dh0, dh0err = zero.clone(), zero.clone()
    for q in range(seqs):
        v, s, e = dfinal[q], dfinal[q].abs(), torch.zeros(c, dtype=torch.float64)
        for t in reversed(range(bounds[q], bounds[q + 1])):
            v, s = v + dy[t], s + dy[t].abs()
            e = e + slack[t] * s
            dx[t], dxerr[t] = b[t] * v, b[t] * e + slack[t] * b[t] * s
            if kind == "decay":
                dg[t], dgsize[t] = v * before[t], s * bsize[t]
                dgerr[t] = s * berr[t] + e * bsize[t] + 4 * U32 * dgsize[t]
            else:
                ab, span = a[t] * b[t], bsize[t] + x[t].abs()
                dg[t], dgsize[t] = ab * v * (before[t] - x[t]), ab * s * span
                dgerr[t] = ab * (s * berr[t] + e * span) + 2 * slack[t] * dgsize[t]
            v, s, e = a[t] * v, a[t].abs() * s, a[t].abs() * e + slack[t] * a[t].abs() * s
        dh0[q], dh0err[q] = v, e
    by_head = lambda t: t.view(n, c // group, group).sum(2)  # noqa: E731
    out.update(dx=(dx, dxerr), dgate=(by_head(dg), by_head(dgerr) + group * U32 * by_head(dgsize)), dh0=(dh0, dh0err))
    return out


def norms(tensors, words, sets):
    squares = [float((t.double().cpu() ** 2).sum()) for t in tensors]
    return torch.tensor([sum(s for s, w in zip(squares, words) if w >> q & 1) for q in range(sets)], dtype=torch.float64).sqrt()


def factors(found, words, max_norm, eps):
    """Per tensor, from the norms as they were found."""
    per = [max_norm / (float(n) + eps) for n in found.double().cpu()]
    out = []
    for w in words:
        mine = [f for q, f in enumerate(per) if w >> q & 1]
        out.append(float("nan") if any(f != f for f in mine) else min([1.0] + mine))
    return out


def adam(p, m, v, g, lr, beta1, beta2, eps, weight_decay, step):
    """((p', error), (m', error), (v', error)) of one tensor, g already scaled (its own relative error: 4 roundings)."""
    p, m, v, g = (t.double().cpu() for t in (p, m, v, g))
    m2, v2 = beta1 * m + (1 - beta1) * g, beta2 * v + (1 - beta2) * g * g
    em = 8 * U32 * (beta1 * m.abs() + (1 - beta1) * g.abs())
    root = (v2 / (1 - beta2 ** step)).sqrt() + eps
    ahead = lr / (1 - beta1 ** step) * m2 / root
    p2 = p - lr * weight_decay * p - ahead
    ep = lr / (1 - beta1 ** step) * em / root + 24 * U32 * ahead.abs() + 4 * U32 * p.abs()
    return (p2, ep), (m2, em), (v2, 16 * U32 * v2)
