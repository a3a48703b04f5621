"""Plain 64-bit forms of the operators of a selective recurrent layer, and how far a 32-bit computation may be off.

As in values_oracle a bound is carried along with the values: for each value S, the sum of the absolute values of all terms
of it, and E, its error; U is half a step of 32 bits.  A product or sum of n terms adds at most n + 1 roundings of S.

The decay exp(d A) with d = softplus(v), v = delta + bias: v is off by U (|delta| + |bias|), which d and the slope (both with a
derivative of at most the slope) pass on; d itself is made with at most 8 roundings, the argument of the exponential with 4 and
the exponential with 6 units.  A strip of up to 64 rows also forms exp(A sum d), whose sum has at most 64 roundings: per row another
64 U |d A|.
"""
import numpy as np
import torch

from values_oracle import U32 as U


def _lengths(rowptr):
    b = rowptr.tolist()
    return list(zip(b[:-1], b[1:]))


def _sigma(v):
    return 1 / (1 + torch.exp(-v))


def conv(x, weight, bias, rowptr, act, state0=None, dy=None, dfinal=None):
    """{name: (value, error)}: y and final, and dx, dweight, dbias and dstate0 if dy is given.  final has no error."""
    d = lambda t: None if t is None else t.double().cpu()  # noqa: E731
    x, w, dy, dfinal, state0 = d(x), d(weight), d(dy), d(dfinal), d(state0)
    (n, c), k = x.shape, w.shape[1]
    b = torch.zeros(c, dtype=torch.float64) if bias is None else d(bias)
    seqs = len(rowptr) - 1
    zero = lambda *s: torch.zeros(*s, dtype=torch.float64)  # noqa: E731
    y, ye, dx, dxe, final = zero(n, c), zero(n, c), zero(n, c), zero(n, c), zero(seqs, k - 1, c)
    ds, dse, dw, dwe, db, dbe = zero(seqs, k - 1, c), zero(seqs, k - 1, c), zero(c, k), zero(c, k), zero(c), zero(c)
    for q, (lo, hi) in enumerate(_lengths(rowptr)):
        m = hi - lo
        seen = torch.cat((zero(k - 1, c) if state0 is None else state0[q], x[lo:hi]))
        final[q] = seen[m:]
        p, s = b.expand(m, c).clone(), b.abs().expand(m, c).clone()
        for j in range(k):
            p, s = p + seen[j:j + m] * w[:, j], s + (seen[j:j + m] * w[:, j]).abs()
        e = (k + 2) * U * s
        y[lo:hi], ye[lo:hi] = p, e
        slope, slope_error = torch.ones_like(p), torch.zeros_like(p)
        if act == "silu":
            g = _sigma(p)
            y[lo:hi], ye[lo:hi] = p * g, 1.1 * e + (p.abs() + 8) * U * (p * g).abs()
            slope = g * (1 + p * (1 - g))
            slope_error = 0.5 * e + (2 * p.abs() + 16) * U * g * (1 + p.abs())
        if dy is None:
            continue
        g = dy[lo:hi] * slope
        ge = dy[lo:hi].abs() * (slope_error + 4 * U * slope.abs())
        grad, error = zero(m + k - 1, c), zero(m + k - 1, c)
        for j in range(k):
            grad[j:j + m] += g * w[:, j]
            error[j:j + m] += (ge + (k + 3) * U * g.abs()) * w[:, j].abs()
            dw[:, j] += (g * seen[j:j + m]).sum(0)
            dwe[:, j] += ((ge + 70 * U * g.abs()) * seen[j:j + m].abs()).sum(0)
        db += g.sum(0)
        dbe += (ge + 70 * U * g.abs()).sum(0)
        if dfinal is not None:
            grad[m:] += dfinal[q]
            error[m:] += 2 * U * dfinal[q].abs()
        dx[lo:hi], dxe[lo:hi], ds[q], dse[q] = grad[k - 1:], error[k - 1:], grad[:k - 1], error[:k - 1]
    out = {"y": (y, ye), "final": (final, torch.zeros_like(final))}
    if dy is not None:
        out.update(dx=(dx, dxe), dweight=(dw, dwe), dbias=(db, dbe), dstate0=(ds, dse))
    return out


def select(x, delta, A, B, C, rowptr, groups=1, D=None, delta_bias=None, z=None, h0=None, dy=None, dfinal=None):
    """{name: (value, error)} of y and final, and of all gradients if dy is given."""
    d = lambda t: None if t is None else t.double().cpu()  # noqa: E731
    x, delta, A, z, dy, dfinal, h0, D, bias = (d(t) for t in (x, delta, A, z, dy, dfinal, h0, D, delta_bias))
    (n, c), N = x.shape, A.shape[1]
    share, seqs = c // groups, len(rowptr) - 1
    full = lambda t: d(t).view(n, groups, 1, N).expand(n, groups, share, N).reshape(n, c, N)  # noqa: E731
    B, C = full(B), full(C)
    zero = lambda *s: torch.zeros(*s, dtype=torch.float64)  # noqa: E731
    bias = zero(c) if bias is None else bias
    v = delta + bias
    slope = _sigma(v)
    slope_error = slope * (2 * U * (delta.abs() + bias.abs()) + 8 * U)
    step = torch.logaddexp(v, torch.zeros_like(v))
    step_error = 2 * slope * U * (delta.abs() + bias.abs()) + 8 * U * step
    a = torch.exp(step[:, :, None] * A)
    slack = A.abs() * step_error[:, :, None] + ((4 + 64) * (step[:, :, None] * A).abs() + 8) * U         # of a, relative
    u, us = (step * x)[:, :, None] * B, (step * x.abs())[:, :, None] * B.abs()
    ue = (step_error * x.abs())[:, :, None] * B.abs() + 4 * U * us
    start = zero(seqs, c, N) if h0 is None else h0
    before, bs, be, h, hs, he = (zero(n, c, N) for _ in range(6))
    final, fe = start.clone(), zero(seqs, c, N)
    for q, (lo, hi) in enumerate(_lengths(rowptr)):
        m, s, e = start[q], start[q].abs(), zero(c, N)
        for t in range(lo, hi):
            before[t], bs[t], be[t] = m, s, e
            m, e, s = a[t] * m + u[t], a[t] * (e + slack[t] * s) + ue[t], a[t] * s + us[t]
            e = e + 2 * U * s
            h[t], hs[t], he[t] = m, s, e
        final[q], fe[q] = m, e
    y, ys = (C * h).sum(2), (C.abs() * hs).sum(2)
    ye = (C.abs() * he).sum(2)
    if D is not None:
        y, ys = y + D * x, ys + (D * x).abs()
    ye = ye + (N + 4) * U * ys
    gate, gr = (torch.ones_like(x), torch.zeros_like(x)) if z is None else (z * _sigma(z), (z.abs() + 8) * U)
    out = {"y": (y * gate, gate.abs() * (ye + gr * ys)), "final": (final, fe)}
    if dy is None:
        return out
    o, oe = dy * gate, (gr + 2 * U) * (dy * gate).abs()
    dfinal = zero(seqs, c, N) if dfinal is None else dfinal
    e, es, ee = (zero(n, c, N) for _ in range(3))
    dh0, dh0e = zero(seqs, c, N), zero(seqs, c, N)
    for q, (lo, hi) in enumerate(_lengths(rowptr)):
        m, s, r = dfinal[q], dfinal[q].abs(), zero(c, N)
        for t in reversed(range(lo, hi)):
            ot = o[t][:, None]
            m, s = m + ot * C[t], s + (ot * C[t]).abs()
            r = r + oe[t][:, None] * C[t].abs() + 2 * U * s
            e[t], es[t], ee[t] = m, s, r
            m, s, r = a[t] * m, a[t] * s, a[t] * (r + (slack[t] + 2 * U) * s)
        dh0[q], dh0e[q] = m, r
    group = lambda t: t.view(n, groups, share, N).sum(2).flatten(1)  # noqa: E731
    ab, k = o.abs()[:, :, None], (share + 8) * U
    dC, dCe = group(o[:, :, None] * h), group(oe[:, :, None] * hs + ab * he + k * ab * hs)
    dxn, xa = (step * x)[:, :, None], x.abs()[:, :, None]
    dB = group(e * dxn)
    dBe = group(ee * dxn.abs() + es * step_error[:, :, None] * xa + k * es * dxn.abs())
    eb, ebs, ebe = (e * B).sum(2), (es * B.abs()).sum(2), (ee * B.abs()).sum(2)
    ebe = ebe + (N + 2) * U * ebs
    skip = zero(c) if D is None else D
    dx = skip * o + step * eb
    dxe = skip.abs() * oe + step * ebe + step_error * ebs + 4 * U * ((skip * o).abs() + step * ebs)
    w, ws = e * a * before, es * a * bs
    we = a * (ee * bs + es * be) + (slack + 3 * U) * ws
    inner, inners = (w * A).sum(2) + eb * x, (ws * A.abs()).sum(2) + ebs * x.abs()
    innere = (we * A.abs()).sum(2) + ebe * x.abs() + (N + 6) * U * inners
    ddelta, dde = inner * slope, slope * innere + (slope_error + 2 * U * slope) * inners
    st, of = step[:, :, None], slice(int(rowptr[0]), int(rowptr[-1]))      # (rows of no sequence do not count)
    total = lambda t: t[of].sum(0)  # noqa: E731
    out.update(dx=(dx, dxe), ddelta=(ddelta, dde), dB=(dB, dBe), dC=(dC, dCe), dh0=(dh0, dh0e),
               dA=(total(w * st), total(we * st + ws * step_error[:, :, None] + 80 * U * ws * st)),
               dD=(total(o * x), total((oe + 80 * U * o.abs()) * x.abs())),
               ddelta_bias=(total(ddelta), total(dde + 80 * U * slope * inners)))
    if z is not None:
        s = _sigma(z)
        dz, room = dy * y * s * (1 + z * (1 - s)), s * (1 + z.abs())
        out["dz"] = (dz, dy.abs() * room * (ye + (2 * z.abs() + 16) * U * ys))
    return out


M0, M1, W0, W1 = 0xD2511F53, 0xCD9E8D57, 0x9E3779B9, 0xBB67AE85


def philox(counter, key, rounds=10):
    """Philox 4x32 with plain integers: counter of four words, key of two -> four words."""
    c, k = list(counter), list(key)
    for _ in range(rounds):
        p, q = M0 * c[0], M1 * c[2]
        c = [(q >> 32) ^ c[1] ^ k[0], q & 0xFFFFFFFF, (p >> 32) ^ c[3] ^ k[1], p & 0xFFFFFFFF]
        k = [(k[0] + W0) & 0xFFFFFFFF, (k[1] + W1) & 0xFFFFFFFF]
    return c


def draws(n, seed, offset):
    """The 16-bit draws of elements 0 .. n-1."""
    out = []
    for block in range(-(-n // 8)):
        words = philox((block & 0xFFFFFFFF, block >> 32, offset & 0xFFFFFFFF, offset >> 32), (seed & 0xFFFFFFFF, seed >> 32))
        out += [part for w in words for part in (w & 0xFFFF, w >> 16)]
    return np.array(out[:n])
