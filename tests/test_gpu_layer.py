"""The operators of a selective recurrent layer together, as a program runs them, and what their owners refuse."""
import pytest
import torch

import layer_oracle as lo
import values_oracle as vo

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.fixture(scope="module")
def dgn():
    assert torch.cuda.is_available(), "these tests need the GPU"
    import paper_1707_08265_amd as d
    return d


class Layer:
    """x -> x + dropout((select(silu(conv(x w_in))) w_out)) over ragged rows, and its gradients, in the given type."""
    C, N, WIDTH = 48, 16, 20

    def __init__(self, dgn, lens, dtype=torch.float32, seed=0):
        gen = torch.Generator().manual_seed(seed)
        rn = lambda *s: torch.randn(*s, generator=gen).cuda()  # noqa: E731
        c, n, w, t, s = self.C, self.N, self.WIDTH, sum(lens), len(lens)
        self.dtype, self.rowptr = dtype, torch.tensor([0] + torch.tensor(lens).cumsum(0).tolist()).cuda()
        self.w = {"w_in": rn(w, 2 * c) / w ** 0.5, "w_bcd": rn(c, 2 * n + c) / c ** 0.5, "w_out": rn(c, w) / c ** 0.5,
                  "conv": rn(c, 4) / 2, "conv_bias": rn(c) * 0.1, "A": -torch.exp(rn(c, n) * 0.5), "D": rn(c), "delta_bias": rn(c) - 2}
        self.key = torch.tensor([seed + 5, 0]).cuda()
        self.conv = dgn.ConvBuffers(t, s, c, dtype=dtype, train=True)
        self.sel = dgn.SelectiveBuffers(t, s, c, num_states=n, dtype=dtype, train=True)
        self.drop = dgn.DropoutBuffers(t, w, 0.25, dtype=dtype)

    def forward(self, x):
        c, n, w = self.C, self.N, {k: v.to(self.dtype) for k, v in self.w.items()}
        both = x @ w["w_in"]
        self.x, self.u, self.z = x, both[:, :c], both[:, c:]                     # (columns of a wider matrix)
        self.conv.forward(self.u, self.w["conv"], self.rowptr, bias=self.w["conv_bias"])
        bcd = self.conv.y @ w["w_bcd"]
        self.i = dict(x=self.conv.y, delta=bcd[:, 2 * n:], A=self.w["A"], B=bcd[:, :n], C=bcd[:, n:2 * n], D=self.w["D"],
                      delta_bias=self.w["delta_bias"], z=self.z, seq_rowptr=self.rowptr)
        self.sel.forward(**self.i)
        self.drop.forward(self.sel.y @ w["w_out"], self.key, residual=x)
        return self.drop.y

    def backward(self, dy):
        w = {k: v.to(self.dtype) for k, v in self.w.items()}
        self.drop.backward(dy, self.key)
        g = {"w_out": self.sel.y.t() @ self.drop.dx}
        self.sel.backward(**self.i, dy=self.drop.dx @ w["w_out"].t())
        s = self.sel
        dbcd = torch.cat((s.dB, s.dC, s.ddelta), 1)
        g["w_bcd"] = self.conv.y.t() @ dbcd
        self.conv.backward(self.u, self.w["conv"], self.rowptr, s.dx + dbcd @ w["w_bcd"].t(), bias=self.w["conv_bias"])
        dboth = torch.cat((self.conv.dx, s.dz), 1)
        g["w_in"] = self.x.t() @ dboth
        g.update(conv=self.conv.dweight, conv_bias=self.conv.dbias, A=s.dA, D=s.dD, delta_bias=s.ddelta_bias)
        return dy + dboth @ w["w_in"].t(), g

    def plain(self, x, w):
        """The layer's outputs in 64 bits on the CPU, for parameters w."""
        c, n, ptr = self.C, self.N, self.rowptr.cpu()
        both = x @ w["w_in"]
        u = lo.conv(both[:, :c], w["conv"], w["conv_bias"], ptr, "silu")["y"][0]
        bcd = u @ w["w_bcd"]
        y = lo.select(u, bcd[:, 2 * n:], w["A"], bcd[:, :n], bcd[:, n:2 * n], ptr, D=w["D"], delta_bias=w["delta_bias"],
                      z=both[:, c:])["y"][0]
        seed, step = self.key.tolist()
        drop = int(0.25 * 65536)
        keep = torch.from_numpy(lo.draws(x.shape[0] * self.WIDTH, seed, step) >= drop).view(x.shape)
        return x + torch.where(keep, (y @ w["w_out"]) * (65536 / (65536 - drop)), 0.0)


def test_the_gradients_of_a_layer_are_its_differences(dgn):
    layer = Layer(dgn, [19, 0, 1, 30])
    gen = torch.Generator().manual_seed(1)
    x, dy = torch.randn(50, layer.WIDTH, generator=gen).cuda(), torch.randn(50, layer.WIDTH, generator=gen).cuda()
    y = layer.forward(x)
    dx, grads = layer.backward(dy)
    w64 = {k: v.double().cpu() for k, v in layer.w.items()}
    want, x64, dy64 = layer.plain(x.double().cpu(), w64), x.double().cpu(), dy.double().cpu()
    # the library's part is exact to some 1e-6 of each value (see the operators' own tests), the products between to 48 half steps
    assert ((y.double().cpu() - want).abs() <= 2e-5 * want.abs().max()).all()
    for name in ["x", *w64]:
        at = x64 if name == "x" else w64[name]
        way = torch.randn(at.shape, generator=gen, dtype=torch.float64)

        def loss(h):
            if name == "x":
                return float((layer.plain(x64 + h * way, w64) * dy64).sum())
            return float((layer.plain(x64, {**w64, name: at + h * way}) * dy64).sum())
        got, each = dx if name == "x" else grads[name], None
        each = got.double().cpu() * way
        # differences of 1e-5 are off by their square, and 32-bit gradients by 2e-5 of each of their terms at most
        assert abs((loss(1e-5) - loss(-1e-5)) / 2e-5 - float(each.sum())) <= 2e-5 * float(each.abs().sum()) + 1e-5, name


def test_a_captured_step_of_a_layer(dgn):
    """Forward and backward in one graph, replayed with other inputs and another step number."""
    layer = Layer(dgn, [70, 0, 33, 200], BF16)
    x, dy = torch.randn(303, layer.WIDTH).to(BF16).cuda(), torch.randn(303, layer.WIDTH).to(BF16).cuda()
    names = {"y": lambda: layer.drop.y, "conv": lambda: layer.conv.dweight, "A": lambda: layer.sel.dA, "dB": lambda: layer.sel.dB,
             "dz": lambda: layer.sel.dz, "ddelta": lambda: layer.sel.ddelta, "conv dx": lambda: layer.conv.dx}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):                   # (the products' own warm-up)
        layer.forward(x)
        layer.backward(dy)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.forward(x)
        layer.backward(dy)
    for k in range(3):
        x.copy_(torch.randn(303, layer.WIDTH).cuda())
        layer.key[1] = k
        graph.replay()
        torch.cuda.synchronize()
        got = {n: f().clone() for n, f in names.items()}
        eager = Layer(dgn, [70, 0, 33, 200], BF16)
        eager.key[1] = k
        eager.forward(x)
        eager.backward(dy)
        for n, v in {"y": eager.drop.y, "conv": eager.conv.dweight, "A": eager.sel.dA, "dB": eager.sel.dB, "dz": eager.sel.dz,
                     "ddelta": eager.sel.ddelta, "conv dx": eager.conv.dx}.items():
            assert torch.equal(got[n], v), (k, n)


def test_a_prompt_and_then_token_by_token(dgn):
    """The states that a prompt ends with, put into pools of both operators, go on as the longer prompt does."""
    c, n, lens, more = 40, 16, [33, 5, 70], 6
    for dtype in (torch.float32, BF16):
        gen = torch.Generator().manual_seed(2)
        rn = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
        total = [v + more for v in lens]
        whole = dict(u=rn(sum(total), c), delta=rn(sum(total), c), B=rn(sum(total), n), C=rn(sum(total), n), z=rn(sum(total), c))
        whole = {k: v.to(dtype).cuda() for k, v in whole.items()}
        w, bias, A = rn(c, 4).cuda(), rn(c).cuda(), -torch.exp(rn(c, n)).cuda()
        starts = [sum(total[:q]) for q in range(3)]
        short = {k: torch.cat([v[s:s + m] for s, m in zip(starts, lens)]) for k, v in whole.items()}
        ptr = lambda ls: torch.tensor([0] + torch.tensor(ls).cumsum(0).tolist()).cuda()  # noqa: E731
        conv, sel = dgn.ConvBuffers(sum(lens), 3, c, dtype=dtype), dgn.SelectiveBuffers(sum(lens), 3, c, num_states=n, dtype=dtype)
        conv.forward(short["u"], w, ptr(lens), bias=bias)
        sel.forward(conv.y, short["delta"], A, short["B"], short["C"], ptr(lens), z=short["z"])
        pools = torch.zeros(5, 3, c, dtype=dtype, device="cuda"), torch.zeros(5, c, n, device="cuda")
        slots = torch.tensor([4, 0, 2], dtype=torch.int32).cuda()
        pools[0][slots.long()], pools[1][slots.long()] = conv.final, sel.final
        cs, ss = dgn.ConvStepBuffers(3, 5, c, dtype=dtype), dgn.SelectiveStepBuffers(3, 5, c, num_states=n, dtype=dtype)
        out, inner = [], []
        for k in range(more):
            at = [s + m + k for s, m in zip(starts, lens)]
            one = {k2: v[at] for k2, v in whole.items()}
            cs.step(one["u"], w, slots, pools[0], bias=bias)
            inner.append(cs.y.clone())
            ss.step(cs.y, one["delta"], A, one["B"], one["C"], slots, pools[1], z=one["z"])
            out.append(ss.y.clone())
        # against the plain forms over the whole; the scan's on the convolution's own outputs
        value, error = lo.conv(whole["u"], w, bias, ptr(total), "silu")["y"]
        seen = torch.cat([torch.cat((conv.y[sum(lens[:q]):sum(lens[:q + 1])], torch.stack([v[q] for v in inner]))) for q in range(3)])
        vo.within(seen, value, error, "convolution")
        want = lo.select(seen, whole["delta"], A, whole["B"], whole["C"], ptr(total), z=whole["z"])
        for q in range(3):
            rows = slice(starts[q] + lens[q], starts[q] + total[q])
            vo.within(torch.stack([v[q] for v in out]), want["y"][0][rows], want["y"][1][rows], "scan")
        vo.within(pools[1][slots.long()], *want["final"], "states")
        assert (pools[0][[1, 3]] == 0).all() and (pools[1][[1, 3]] == 0).all()


@pytest.mark.parametrize("states,groups", [(16, 1), (16, 3), (8, 1), (4, 1), (64, 2), (128, 1), (256, 1), (12, 1)])
def test_one_token_for_many_rows(dgn, states, groups):
    """Enough rows that a wave takes several blocks of channels, with blocks that end inside a wave's, and states past the caches."""
    c, rows = 276 // groups * groups, 700 if states <= 64 else 300
    gen = torch.Generator(device="cuda").manual_seed(states)
    rn = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    for dtype, more in [(BF16, 1), (torch.float32, 3)]:
        n = rows * more
        i = dict(x=rn(n, c).to(dtype), delta=rn(n, c).to(dtype), A=-torch.exp(rn(c, states)), B=rn(n, groups * states).to(dtype),
                 C=rn(n, groups * states).to(dtype), D=rn(c), delta_bias=rn(c) - 2, z=rn(n, c).to(dtype))
        pool = rn(n + 9, c, states)
        slots = torch.randperm(n + 9, generator=gen, device="cuda")[:n].to(torch.int32)
        slots[5::50] = -1
        b = dgn.SelectiveStepBuffers(n, n + 9, c, num_states=states, num_groups=groups, dtype=dtype)
        print(f"select step: {n} rows of {c} x {states} in {groups}, {dtype}", flush=True)
        out = pool.clone()
        b.step(**i, slots=slots, state_in=pool, state_out=out)
        some = torch.tensor([0, 1, 5, n // 2, n - 2, n - 1])
        for r in some.tolist():
            s = int(slots[r])
            if s < 0:
                assert (b.y[r] == 0).all()
                continue
            one = {k: v[r:r + 1] if k in ("x", "delta", "B", "C", "z") else v for k, v in i.items()}
            want = lo.select(**one, rowptr=torch.tensor([0, 1]), groups=groups, h0=pool[s:s + 1])
            vo.within(b.y[r:r + 1], *want["y"], "y")
            vo.within(out[s:s + 1], *want["final"], "state")
        idle = torch.ones(n + 9, dtype=torch.bool, device="cuda")
        idle[slots[slots >= 0].long()] = False
        assert torch.equal(out[idle], pool[idle]) and not torch.equal(out[~idle], pool[~idle])
        # every row against the plain form in 32 bits, to 4 000 half steps of its largest terms
        live = slots >= 0
        d = torch.nn.functional.softplus(i["delta"][live].float() + i["delta_bias"])
        wide = lambda t: t[live].float().view(-1, groups, 1, states).expand(-1, -1, c // groups, -1).reshape(-1, c, states)  # noqa: E731
        h = torch.exp(d[:, :, None] * i["A"]) * pool[slots[live].long()] + (d * i["x"][live].float())[:, :, None] * wide(i["B"])
        assert ((out[slots[live].long()] - h).abs() <= 4000 * vo.U32 * h.abs().max()).all()


def test_offsets_past_32_bits(dgn):
    """Rows 2^28 elements apart: the last ones past 2^32 elements."""
    rows, c, n, t = 18, 24, 16, BF16
    far = torch.empty(rows, 1 << 28, dtype=t, device="cuda")
    put = lambda k, v: far[:, 1000 * k:1000 * k + v.shape[1]].copy_(v)  # noqa: E731
    gen = torch.Generator(device="cuda").manual_seed(4)
    rn = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    x, dy, delta, z, B, C = (put(k, rn(rows, w).to(t)) for k, w in enumerate((c, c, c, c, n, n)))
    ptr, w, A = torch.tensor([0, 11, 18]).cuda(), rn(c, 4), -torch.exp(rn(c, n))
    conv = dgn.ConvBuffers(rows, 2, c, dtype=t, train=True)
    conv.forward(x, w, ptr)
    conv.backward(x, w, ptr, dy)
    for name, (value, error) in lo.conv(x, w, None, ptr, "silu", dy=dy).items():
        if name not in ("dbias", "dstate0", "final"):
            vo.within(getattr(conv, name), value, error, name)
    sel = dgn.SelectiveBuffers(rows, 2, c, num_states=n, dtype=t, train=True)
    sel.forward(x, delta, A, B, C, ptr, z=z)
    sel.backward(x, delta, A, B, C, ptr, dy, z=z)
    for name, (value, error) in lo.select(x, delta, A, B, C, ptr, z=z, dy=dy).items():
        vo.within(getattr(sel, name), value, error, name)
    drop = dgn.DropoutBuffers(rows, c, 0.5, dtype=t)
    drop.forward(x, torch.tensor([1, 2]).cuda(), residual=dy)
    keep = torch.from_numpy(lo.draws(rows * c, 1, 2) >= 32768).view(rows, c)
    want = torch.where(keep, 2 * x.double().cpu(), 0.0) + dy.double().cpu()
    vo.within(drop.y, want, 4 * vo.U32 * want.abs(), "dropout")


def test_owners_refuse_other_shapes_types_and_places(dgn):
    c, n, t, s = 8, 4, 6, 2
    x, f = torch.zeros(t, c, dtype=BF16, device="cuda"), lambda *v: torch.zeros(*v, device="cuda")
    ptr, w, shared = torch.tensor([0, 2, 6]).cuda(), f(c, 4), torch.zeros(t, n, dtype=BF16, device="cuda")
    conv, sel = dgn.ConvBuffers(t, s, c, train=True), dgn.SelectiveBuffers(t, s, c, num_states=n, train=True)
    cs, ss = dgn.ConvStepBuffers(t, 3, c), dgn.SelectiveStepBuffers(t, 3, c, num_states=n)
    drop, key = dgn.DropoutBuffers(t, c, 0.5), torch.tensor([1, 2]).cuda()
    slots = torch.zeros(t, dtype=torch.int32, device="cuda")
    pool = torch.zeros(3, 3, c, dtype=BF16, device="cuda")
    calls = {
        "conv": (conv.forward, dict(x=x, weight=w, seq_rowptr=ptr, bias=f(c), state0=torch.zeros(s, 3, c, dtype=BF16, device="cuda"))),
        "conv back": (conv.backward, dict(x=x, weight=w, seq_rowptr=ptr, dy=x)),
        "conv step": (cs.step, dict(x=x, weight=w, slots=slots, state_in=pool)),
        "select": (sel.forward, dict(x=x, delta=x, A=f(c, n), B=shared, C=shared, seq_rowptr=ptr, D=f(c), delta_bias=f(c), z=x, h0=f(s, c, n))),
        "select back": (sel.backward, dict(x=x, delta=x, A=f(c, n), B=shared, C=shared, seq_rowptr=ptr, dy=x, dfinal=f(s, c, n))),
        "select step": (ss.step, dict(x=x, delta=x, A=f(c, n), B=shared, C=shared, slots=slots, state_in=f(3, c, n), z=x)),
        "dropout": (drop.forward, dict(x=x, key=key, residual=x)),
        "dropout back": (drop.backward, dict(dy=x, key=key)),
    }
    other = torch.cuda.Stream()
    for what, (call, good) in calls.items():
        for name, v in good.items():
            for bad in (v.cpu(), v.double(), v[:-1] if v.dim() else v, torch.cat((v, v), -1), v.tolist()):
                with pytest.raises(dgn.DgnError):
                    call(**{**good, name: bad})
        if what.endswith("step"):
            slots.copy_(torch.tensor([0, 1, 2, -1, -1, -1]))
        with torch.cuda.stream(other):
            other.wait_stream(torch.cuda.default_stream())
            call(**good)
        call(**good, stream=other)
        other.synchronize()
    with pytest.raises(dgn.DgnError):
        conv.backward(x, w, ptr, x, state0=conv.final)
    with pytest.raises(dgn.DgnError):
        sel.backward(x, x, f(c, n), shared, shared, ptr, x, h0=sel.final)
    for call in (dgn.ConvBuffers(t, s, c).backward, ):
        with pytest.raises(dgn.DgnError):
            call(x, w, ptr, x)
    with pytest.raises(dgn.DgnError):
        dgn.SelectiveBuffers(t, s, c, num_states=n).backward(x, x, f(c, n), shared, shared, ptr, x)


def test_row_pointers_outside_and_out_of_order(dgn):
    """Values mean nothing then, but nothing outside is touched: guards around every output."""
    t, s, c, n = 100, 5, 20, 16
    gen = torch.Generator().manual_seed(0)
    room = lambda shape, dtype=BF16: torch.full((shape[0] + 8, *shape[1:]), 7.0, dtype=dtype, device="cuda")  # noqa: E731
    for ptr in ([-50, 10, 300, 40, 2**40, 60], [90, 70, 50, 30, 10, 0], [0, 0, 0, 0, 0, 0], [100, 100, 200, -1, 100, 3]):
        x = torch.randn(t, c, generator=gen).to(BF16).cuda()
        shared, A, w = torch.randn(t, n, generator=gen).to(BF16).cuda(), -torch.ones(c, n, device="cuda"), torch.ones(c, 4, device="cuda")
        p = torch.tensor(ptr).cuda()
        conv, sel = dgn.ConvBuffers(t, s, c, train=True), dgn.SelectiveBuffers(t, s, c, num_states=n, train=True)
        guards = []
        for b, names in ((conv, ("y", "final", "dx", "dstate0", "dweight")), (sel, ("y", "final", "dx", "ddelta", "dB", "dC", "dz", "dA", "dh0"))):
            for name in names:
                old = getattr(b, name)
                full = room(old.shape, old.dtype)
                guards.append((name, full))
                setattr(b, name, full[4:-4])
        sel._grads = dgn.dgn_select_grads(*(v.data_ptr() for v in (sel.dx, sel.ddelta, sel.dA, sel.dB, sel.dC, sel.dD, sel.ddelta_bias,
                                                                   sel.dz, sel.dh0)))
        conv.forward(x, w, p)
        conv.backward(x, w, p, x)
        sel.forward(x, x, A, shared, shared, p, z=x)
        sel.backward(x, x, A, shared, shared, p, x, z=x)
        torch.cuda.synchronize()
        for name, full in guards:
            assert (full[:4] == 7.0).all() and (full[-4:] == 7.0).all(), (ptr, name)
