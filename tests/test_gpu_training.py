"""The training step of a network of micro-DAG blocks: norms, DAGs, loss and updates together."""
import pytest
import torch
import torch.nn.functional as F

import operators_ref as ref
from paper_2304_07741_amd import training

pytestmark = pytest.mark.gpu

SHAPE, CLASSES, GROUPS = (6, 32, 7, 9), 11, 4


def _reference(net, x, labels, entropy_weight):
    """The same network in 64 bits with autograd; returns (loss, logits, leaves by name)."""
    n, c, h, w = SHAPE
    leaf = lambda t: t.detach().double().cpu().requires_grad_()  # noqa: E731
    leaves = {"x": leaf(x)}
    for i, v in enumerate(net.vectors):
        leaves |= {f"{k}{i}": leaf(t) for k, t in v.items()}
    for name, dags in (("block", net.blocks), ("gate", net.gates), ("head", [net.head])):
        leaves |= {f"{name}{i}": leaf(d.run.w[0]) for i, d in enumerate(dags)}
    col = lambda t: t[None, :, None, None]  # noqa: E731
    rms = lambda t: t * ((t * t).mean(1, keepdim=True) + 1e-6) ** -0.5  # noqa: E731
    xs = leaves["x"]
    u = rms(xs) * col(leaves["w_pre0"])
    for i in range(len(net.blocks)):
        z = F.gelu(F.conv2d(u, leaves[f"block{i}"].reshape(c, c // GROUPS, 3, 3), padding=1, groups=GROUPS))
        g = F.conv2d(u, leaves[f"gate{i}"].reshape(c, c, 1, 1))
        xs = xs + col(leaves[f"scale{i + 1}"]) * F.silu(g) * rms(z) * col(leaves[f"w_post{i + 1}"])
        u = rms(xs) * col(leaves[f"w_pre{i + 1}"])
    logits = u.mean((2, 3)) @ leaves["head0"][0].T
    logp = F.log_softmax(logits, 1)
    entropy = -(logp.exp() * logp).sum(1)
    loss = -logp[torch.arange(n), labels.cpu()].mean() - entropy_weight * entropy.mean()
    loss.backward()
    return float(loss.detach()), logits, leaves


@pytest.mark.parametrize("dtype,tol", [("f32", 1e-4), ("bf16", 5e-2)])
def test_gradients_of_the_whole_step(dtype, tol):
    """fp32: the 1e-5 of each of some ten stages in a row; bf16: 2^-9 per stored map through as many stages, and 2e-2 of the DAGs."""
    net = training.BlockNet(SHAPE, CLASSES, 2, dtype, GROUPS)
    x, labels = training.synthetic(SHAPE[0], SHAPE, CLASSES, net.first.tdtype, 3)
    net.forward(x)
    scores = {k: v.clone() for k, v in net.scores(labels).items()}
    dx = net.backward(labels, 0.1)
    loss, logits, leaves = _reference(net, x, labels, 0.1)
    got = {"x": dx, **{f"block{i}": d.run.dw[0] for i, d in enumerate(net.blocks)}, **{f"gate{i}": d.run.dw[0] for i, d in enumerate(net.gates)},
           "head0": net.head.run.dw[0]}
    for i, v in enumerate(net.dvectors):
        got |= {f"{k}{i}": t for k, t in v.items()}
    mine = float((-scores["logprob"] - 0.1 * scores["entropy"]).double().mean())
    assert abs(mine - loss) <= tol * abs(loss)
    for k, t in got.items():
        want, have = leaves[k].grad, t.double().cpu().reshape(leaves[k].shape)
        assert float((have - want).norm()) <= tol * float(want.norm()), k
    net.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_update_is_the_orthogonalised_momentum(dtype):
    net = training.BlockNet(SHAPE, CLASSES, 1, dtype, GROUPS)
    x, labels = training.synthetic(SHAPE[0], SHAPE, CLASSES, net.first.tdtype, 5)
    d = net.blocks[0]
    m = torch.zeros_like(d.momentum[0], dtype=torch.float64, device="cpu")
    w = d.master[0].double().cpu()
    for _ in range(3):
        net.forward(x)
        net.backward(labels)
        want = ref.ortho_step(d.run.dw[0].double().cpu(), m, 0.9, True, 5, w, 0.02)
        net.update(lr=0.02, mu=0.9)
        m, w = want["momentum"], want["master"]
        assert float((d.master[0].double().cpu() - w).norm()) <= 1e-4 * float(w.norm())
        assert torch.equal(d.run.w[0], d.master[0].to(d.run.w[0].dtype))
    net.close()


def test_the_loss_falls():
    net = training.BlockNet((32, 32, 8, 8), 10, 2, "bf16")
    losses = []
    for step in range(40):
        x, labels = training.synthetic(32, (32, 32, 8, 8), 10, torch.bfloat16, step)
        net.forward(x)
        losses.append(float(-net.scores(labels)["logprob"].mean()))
        net.backward(labels)
        net.update()
    net.close()
    assert sum(losses[-5:]) < 0.5 * sum(losses[:5]), losses
