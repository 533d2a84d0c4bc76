"""A small network of micro-DAG blocks and its training step, in the library's kernels throughout:

    u_0 = norm(x_0)                                     canvas_norm, PRE
    z_i = block(u_{i-1}), g_i = gate(u_{i-1})           canvas_dag (the block's template, one FC for the gate)
    x_i = x_{i-1} + scale silu(g_i) norm(z_i)           canvas_norm, POST and PRE in one launch
    u_i = norm(x_i)
    logits = FC(mean over the pixels of u_L)            canvas_dag
    loss = mean of -log p(label) - entropy_weight * entropy      canvas_logprob
    W = W - lr * orthogonalised momentum                canvas_ortho, on the fp32 gradients of every FC

torch supplies device memory, adds the two gradients that meet at u_i and updates the norms' weights (vectors of C).

    python -m paper_2304_07741_amd.training [--steps 60] [--dtype bf16]

trains it on synthetic images, each class its levels and a pattern under noise, and prints the loss, the share of labels that are the first of the
three best alternatives, and the share that are among them.
"""
import argparse
import math

import torch

from . import binding as B
from . import harness

BOTH = B.CANVAS_NORM_POST | B.CANVAS_NORM_PRE


def block_text(C, groups=4):
    """3x3 window, grouped FC, GELU: the template of the blocks."""
    return (f"canvas-dag 1\n%1 = unfold %0 kh=3 kw=3\n%2 = fc %1 groups={groups} out={C}\n%3 = unary %2 op=gelu\noutput %3\n")


def gate_text(C):
    return f"canvas-dag 1\n%1 = fc %0 groups=1 out={C}\noutput %1\n"


def head_text(classes):
    return f"canvas-dag 1\n%1 = fold %0 op=avg axis=HW\n%2 = fc %1 groups=1 out={classes}\noutput %2\n"


class _Dag:
    """One micro-DAG of the network: its runner, and per FC weight the fp32 master, the momentum and the update's plan."""

    def __init__(self, text, shape, dtype, generator):
        self.run = harness.DagRunner(text, shape, dtype)
        self.master, self.momentum, self.ortho = [], [], []
        for w, s in zip(self.run.w, self.run.wshapes):
            self.master.append(torch.randn(s, generator=generator, device=w.device) / math.sqrt(s[2]))
            self.momentum.append(torch.zeros(s, device=w.device))
            self.ortho.append(harness.OrthoRunner(s, dtype, flags=B.CANVAS_ORTHO_NESTEROV))
            w.copy_(self.master[-1])

    def forward(self, x):
        r = self.run
        B.canvas_dag_forward(r.handle, x, r.w, r.y, r.ws)
        return r.y

    def backward(self, x, dy):
        r = self.run
        B.canvas_dag_backward(r.handle, x, r.w, dy, r.dx, r.dw, r.ws)
        return r.dx

    def update(self, lr, mu):
        """Momentum and master weights stay in the update's own buffers; the DAG reads the weights that it leaves."""
        for k, o in enumerate(self.ortho):
            R, K = o.shape[1:]
            out = o.step(self.run.dw[k], self.momentum[k], self.master[k], mu=mu, lr=lr * math.sqrt(max(1.0, R / K)))
            self.momentum[k], self.master[k], self.run.w[k] = out["momentum"], out["master"], out["weights"]

    def close(self):
        self.run.close()
        for o in self.ortho:
            o.close()


class BlockNet:
    def __init__(self, shape, classes, depth=2, dtype="bf16", groups=4, seed=0):
        self.shape, self.classes = tuple(int(v) for v in shape), int(classes)
        n, c = self.shape[:2]
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        self.blocks = [_Dag(block_text(c, groups), self.shape, dtype, gen) for _ in range(depth)]
        self.gates = [_Dag(gate_text(c), self.shape, dtype, gen) for _ in range(depth)]
        self.head = _Dag(head_text(classes), self.shape, dtype, gen)
        self.first = harness.NormRunner(self.shape, dtype, B.CANVAS_NORM_PRE)
        self.norms = [harness.NormRunner(self.shape, dtype, BOTH, gate=B.CANVAS_GATE_SILU) for _ in range(depth)]
        self.loss = harness.LogprobRunner(n, classes, dtype, top_k=min(3, classes))
        ones = lambda: torch.ones(c, device="cuda")  # noqa: E731
        self.vectors = [{"w_pre": ones()}] + [{"w_post": ones(), "scale": 0.3 * ones(), "w_pre": ones()} for _ in range(depth)]

    def forward(self, x):
        """logits [N, classes]"""
        u = self.first.forward(x, w_pre=self.vectors[0]["w_pre"])["u"]
        self.inputs, self.xs = [u], [x]
        for block, gate, norm, v in zip(self.blocks, self.gates, self.norms, self.vectors[1:]):
            z, g = block.forward(u).view(self.shape), gate.forward(u).view(self.shape)
            out = norm.forward(self.xs[-1], z, g, v["w_post"], v["scale"], v["w_pre"])
            u = out["u"]
            self.inputs.append(u)
            self.xs.append(out["x_out"])
        self.logits = self.head.forward(u).view(self.shape[0], self.classes)
        return self.logits

    def scores(self, labels):
        """What the loss is made of, and the alternatives: the buffers of the loss's runner."""
        return self.loss.forward(self.logits, labels)

    def backward(self, labels, entropy_weight=0.0):
        """Gradients of mean(-log p(label) - entropy_weight * entropy): in the DAGs' dw, and of the norms' vectors in self.dvectors."""
        n = self.shape[0]
        full = lambda v: torch.full((n,), v, device="cuda")  # noqa: E731
        dlogits = self.loss.backward(self.logits, labels, full(-1.0 / n), full(-entropy_weight / n))["dlogits"]
        du = self.head.backward(self.inputs[-1], dlogits)
        dx, self.dvectors = None, [None] * len(self.vectors)
        for i in range(len(self.blocks), 0, -1):
            block, gate, norm, v = self.blocks[i - 1], self.gates[i - 1], self.norms[i - 1], self.vectors[i]
            z, g = block.run.y.view(self.shape), gate.run.y.view(self.shape)
            grads = norm.backward(self.xs[i], z, g, v["w_post"], v["scale"], v["w_pre"], dx_out=dx, du=du)
            dx = grads["dx"]
            self.dvectors[i] = {k: grads["d" + k] for k in v}
            du = block.backward(self.inputs[i - 1], grads["dz"]) + gate.backward(self.inputs[i - 1], grads["dgate"])
        grads = self.first.backward(self.xs[0], w_pre=self.vectors[0]["w_pre"], dx_out=dx, du=du)
        self.dvectors[0] = {"w_pre": grads["dw_pre"]}
        return grads["dx"]

    def update(self, lr=0.05, mu=0.9):
        for d in [*self.blocks, *self.gates, self.head]:
            d.update(lr, mu)
        for v, dv in zip(self.vectors, self.dvectors):
            for k in v:
                v[k] -= lr * dv[k]

    def close(self):
        for d in [*self.blocks, *self.gates, self.head, self.first, *self.norms, self.loss]:
            d.close()


def synthetic(n, shape, classes, dtype, seed):
    """Images whose class is a fixed random level per channel and a pattern around it, under noise three times as strong."""
    _, c, h, w = shape
    fixed = torch.Generator(device="cuda")
    fixed.manual_seed(1234)
    patterns = torch.randn(classes, c, h, w, generator=fixed, device="cuda") + torch.randn(classes, c, 1, 1, generator=fixed, device="cuda")
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    labels = torch.randint(0, classes, (n,), generator=gen, device="cuda")
    x = patterns[labels] + 3 * torch.randn(n, c, h, w, generator=gen, device="cuda")
    return x.to(dtype), labels


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--dtype", choices=("f32", "bf16"), default="bf16")
    ap.add_argument("--batch", type=int, default=64)
    ap.add_argument("--channels", type=int, default=64)
    ap.add_argument("--side", type=int, default=14)
    ap.add_argument("--classes", type=int, default=100)
    ap.add_argument("--depth", type=int, default=2)
    a = ap.parse_args()
    shape = (a.batch, a.channels, a.side, a.side)
    net = BlockNet(shape, a.classes, a.depth, a.dtype)
    for step in range(a.steps):
        x, labels = synthetic(a.batch, shape, a.classes, net.first.tdtype, step)
        net.forward(x)
        s = net.scores(labels)
        if step % 10 == 0 or step == a.steps - 1:
            hits = s["top_index"] == labels[:, None]
            print(f"step {step:4d}  loss {float(-s['logprob'].mean()):.4f}  entropy {float(s['entropy'].mean()):.4f}  "
                  f"first {float(hits[:, 0].float().mean()):.2f}  among three {float(hits.any(1).float().mean()):.2f}", flush=True)
        net.backward(labels)
        net.update()
    net.close()


if __name__ == "__main__":
    main()
