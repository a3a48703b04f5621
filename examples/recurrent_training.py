"""A training step of a gated recurrent layer, run from its pruned graph.

The step is recorded once as a graph of operators: the layer, the loss, then the gradient operators in inverse order.  Two
functions are solved on it in one prune, as two target sets:

  set 0  "all":   the gradients of all parameters
  set 1  "head":  the gradient of the output projection alone (the rest of the network is frozen)

and each runs its own surviving operators, in creation order.  The updater then takes the prune's tensor mask as it is: norms
of the gradients per set, and an Adam step with clipping that leaves alone what the chosen set does not need.  At the end the
trained layer goes on token by token from the states that the sequences ended with.

Run: python examples/recurrent_training.py   (needs a GPU; prints the losses)
"""
import os
import sys
from types import SimpleNamespace

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1707_08265_amd as dgn  # noqa: E402

WIDTH, CHANNELS, OUT = 48, 160, 16
LENGTHS = [700, 1, 0, 333, 1291, 64]
BF16 = torch.bfloat16


class Program:
    """Operators in the order of their creation, over numbered tensors."""

    def __init__(self):
        self.names, self.ops = {}, []

    def tensor(self, name):
        return self.names.setdefault(name, len(self.names))

    def op(self, run, reads, writes):
        self.ops.append((run, [self.tensor(n) for n in reads.split()], [self.tensor(n) for n in writes.split()]))

    def graph(self):
        pairs = lambda k: [(o, t) for o, op in enumerate(self.ops) for t in op[k]]  # noqa: E731
        ins, outs = pairs(1), pairs(2)
        col = lambda p, i: np.array([e[i] for e in p], dtype=np.int32)  # noqa: E731
        return dgn.DeviceGraph.from_coo(SimpleNamespace(
            num_ops=len(self.ops), num_tensors=len(self.names), in_op=col(ins, 0), in_tensor=col(ins, 1), out_op=col(outs, 0),
            out_tensor=col(outs, 1), num_graphs=1, graph_op_offsets=None, graph_tensor_offsets=None), validate=True)


def record(v, scan, rowptr):
    """The step as a program over the values in ``v`` (name -> tensor)."""
    p = Program()

    def product(a, b, out):
        def run():
            v[out] = v[a] @ v[b]
        p.op(run, f"{a} {b}", out)

    def transposed(a, b, out, left):
        """out = a^T b (left) or a b^T, into the gradient's own memory where it has one."""
        def run():
            x, y = (v[a].t(), v[b]) if left else (v[a], v[b].t())
            if out in v:
                torch.mm(x, y, out=v[out])
            else:
                v[out] = x @ y
        p.op(run, f"{a} {b}", out)

    def recurrence():
        scan.forward(v["z"], v["gate"], rowptr)
        v["h"] = scan.y

    def loss():
        v["dout"] = v["out"].float() - v["target"]
        v["loss"] = v["dout"].square().mean()
        v["dout"] = (v["dout"] * (2.0 / v["dout"].numel())).to(BF16)

    def recurrence_gradient():
        scan.backward(v["z"], v["gate"], rowptr, v["dh"])
        v["dz"], v["dgate"] = scan.dx, scan.dgate

    product("x", "w_in", "z")
    product("x", "w_gate", "gate")
    p.op(recurrence, "z gate", "h")
    product("h", "w_out", "out")
    p.op(loss, "out target", "loss dout")
    transposed("h", "dout", "dw_out", True)             # the gradient operators, in inverse order
    transposed("dout", "w_out", "dh", False)
    p.op(recurrence_gradient, "z gate dh", "dz dgate")
    transposed("x", "dgate", "dw_gate", True)
    transposed("x", "dz", "dw_in", True)
    return p


def run(steps=60, head_steps=10, seed=0, log=print):
    torch.manual_seed(seed)
    tokens, params = sum(LENGTHS), ("w_in", "w_gate", "w_out")
    shapes = {"w_in": (WIDTH, CHANNELS), "w_gate": (WIDTH, CHANNELS), "w_out": (CHANNELS, OUT)}
    new = lambda name, scale: torch.randn(*shapes[name], device="cuda") * scale / shapes[name][0] ** 0.5  # noqa: E731
    rowptr = torch.tensor([0] + np.cumsum(LENGTHS).tolist(), device="cuda")
    scan = dgn.ScanBuffers(tokens, len(LENGTHS), CHANNELS, kind="sigmoid", dtype=BF16, train=True)

    # what is to be learnt: the outputs of another layer of the same kind
    v = {"x": torch.randn(tokens, WIDTH, device="cuda").to(BF16)}
    teach = {n: new(n, 2.0).to(BF16) for n in params}
    scan.forward(v["x"] @ teach["w_in"], v["x"] @ teach["w_gate"], rowptr)
    v["target"] = (scan.y @ teach["w_out"]).float()

    # parameters and moments in 32 bits, the copies and gradients that the operators use in 16
    master = {n: new(n, 1.0) for n in params}
    v.update({n: master[n].to(BF16) for n in params})
    v.update({f"d{n}": torch.zeros(*shapes[n], dtype=BF16, device="cuda") for n in params})
    program = record(v, scan, rowptr)
    graph = program.graph()

    targets = [["dw_in", "dw_gate", "dw_out", "loss"], ["dw_out", "loss"]]
    flat = torch.tensor([program.names[n] for t in targets for n in t], dtype=torch.int32, device="cuda")
    ptr = torch.tensor([0, len(targets[0]), flat.numel()], dtype=torch.int32, device="cuda")
    pruned = dgn.PruneBuffers(graph, len(targets))
    dgn_rc = pruned.prune(ptr, flat)
    assert dgn_rc == 0, dgn.dgn_strerror(dgn_rc)
    lists = dgn.ReadoutBuffers(pruned)
    assert lists.per_set_lists() == 0
    bounds, ops = lists.set_rowptr.tolist(), lists.set_ops.tolist()
    functions = [ops[bounds[q]:bounds[q + 1]] for q in range(len(targets))]
    log(f"{len(program.ops)} operators recorded; 'all' runs {len(functions[0])}, 'head' {len(functions[1])}")

    grads = dgn.TensorList([v[f"d{n}"] for n in params])
    ids = torch.tensor([program.names[f"d{n}"] for n in params], dtype=torch.int32, device="cuda")
    moments = [[torch.zeros_like(master[n]) for n in params] for _ in "mv"]
    norms = dgn.GradientBuffers(grads, len(targets))
    adam = dgn.AdamBuffers(grads, dgn.TensorList([master[n] for n in params]), *(dgn.TensorList(m) for m in moments),
                           copy=dgn.TensorList([v[n] for n in params]))
    masks = [pruned.tensor_mask & (1 << q) for q in range(len(targets))]       # what set q alone needs

    losses, before = [], None
    for step in range(1, steps + head_steps + 1):
        q = 0 if step <= steps else 1
        if step == steps + 1:
            before = {n: master[n].clone() for n in params}
        for o in functions[q]:
            program.ops[o][0]()
        norms.norm(masks[q], ids)
        adam.step(lr=2e-2, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.0, step=step, norms=norms.norms, max_norm=1.0,
                  mask=masks[q], ids=ids, skip_nonfinite=True)
        losses.append(v["loss"])
    losses = [float(x) for x in losses]
    log("loss: " + " ".join(f"{x:.4f}" for x in losses[::10]))

    # one token for each sequence, from the states that they ended with; an idle row in the batch
    scan.forward(v["x"] @ v["w_in"], v["x"] @ v["w_gate"], rowptr)
    pool = scan.final.clone()
    rows = torch.tensor([4, 0, -1, 3], dtype=torch.int32, device="cuda")
    served = dgn.ScanStepBuffers(len(rows), len(LENGTHS), CHANNELS, kind="sigmoid", dtype=BF16)
    x = torch.randn(len(rows), WIDTH, device="cuda").to(BF16)
    served.step(x @ v["w_in"], x @ v["w_gate"], rows, pool)
    answer = served.y @ v["w_out"]
    return SimpleNamespace(losses=losses, before=before, after=master, names=program.names, mask=pruned.tensor_mask, answer=answer,
                           functions=functions, pool=pool, final=scan.final, rows=rows)


if __name__ == "__main__":
    run()
