"""The training step with a gated pair, a head without logits and clipped gradients: all of them together, as a training program runs them."""
import math

import pytest
import torch
import torch.nn.functional as F

import more_operators_ref as ref
import operators_ref
from paper_2304_07741_amd import training

pytestmark = pytest.mark.gpu

SHAPE, CLASSES, GROUPS, WIDE = (6, 32, 7, 9), 11, 4, 40


def _reference(net, x, labels, entropy_weight):
    """The same network in 64 bits with autograd; returns (loss, leaves by name)."""
    n, c, h, w = SHAPE
    leaf = lambda t: t.detach().double().cpu().requires_grad_()  # noqa: E731
    leaves = {"x": leaf(x)}
    for i, v in enumerate(net.vectors):
        leaves |= {f"{k}{i}": leaf(t) for k, t in v.items()}
    for name, dags in (("block", net.blocks), ("gate", net.gates)):
        leaves |= {f"{name}{i}": leaf(d.run.w[0]) for i, d in enumerate(dags)}
    leaves |= {f"wide{i}": leaf(t) for i, t in enumerate(net.wide.weights)}
    col = lambda t: t[None, :, None, None]  # noqa: E731
    rms = lambda t: t * ((t * t).mean(1, keepdim=True) + 1e-6) ** -0.5  # noqa: E731
    xs = leaves["x"]
    u = rms(xs) * col(leaves["w_pre0"])
    for i in range(len(net.blocks)):
        z = F.gelu(F.conv2d(u, leaves[f"block{i}"].reshape(c, c // GROUPS, 3, 3), padding=1, groups=GROUPS))
        g = F.conv2d(u, leaves[f"gate{i}"].reshape(c, c, 1, 1))
        xs = xs + col(leaves[f"scale{i + 1}"]) * F.silu(g) * rms(z) * col(leaves[f"w_post{i + 1}"])
        u = rms(xs) * col(leaves[f"w_pre{i + 1}"])
    p = u.mean((2, 3))
    v = F.silu(p @ leaves["wide0"].T) * (p @ leaves["wide1"].T)
    logp = F.log_softmax(v @ leaves["wide2"].T, 1)
    entropy = -(logp.exp() * logp).sum(1)
    loss = -logp[torch.arange(n), labels.cpu()].mean() - entropy_weight * entropy.mean()
    loss.backward()
    return float(loss.detach()), leaves


def _net(dtype, **k):
    net = training.BlockNet(SHAPE, CLASSES, 2, dtype, GROUPS, widen=WIDE, **k)
    x, labels = training.synthetic(SHAPE[0], SHAPE, CLASSES, net.first.tdtype, 3)
    return net, x, labels


@pytest.mark.parametrize("dtype,tol", [("f32", 1e-4), ("bf16", 5e-2)])
def test_gradients_of_the_whole_step(dtype, tol):
    """fp32: the 1e-5 of each of some twelve stages in a row; bf16: 2^-8 per stored map or row through as many stages, and 2e-2 of the DAGs."""
    net, x, labels = _net(dtype)
    net.forward(x)
    scores = {k: v.clone() for k, v in net.scores(labels).items()}
    dx = net.backward(labels, 0.1)
    loss, leaves = _reference(net, x, labels, 0.1)
    got = {"x": dx, **{f"block{i}": d.run.dw[0] for i, d in enumerate(net.blocks)}, **{f"gate{i}": d.run.dw[0] for i, d in enumerate(net.gates)},
           **{f"wide{i}": g for i, g in enumerate(net.wide.grads)}}
    for i, v in enumerate(net.dvectors):
        got |= {f"{k}{i}": t for k, t in v.items()}
    mine = float((-scores["logprob"] - 0.1 * scores["entropy"]).double().mean())
    assert abs(mine - loss) <= tol * abs(loss)
    for k, t in got.items():
        want, have = leaves[k].grad, t.double().cpu().reshape(leaves[k].shape)
        assert float((have - want).norm()) <= tol * float(want.norm()), k
    net.close()


@pytest.mark.parametrize("max_norm", [None, 0.05, 1e6])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_updates_take_the_clipped_gradients(dtype, max_norm):
    net, x, labels = _net(dtype, max_norm=max_norm)
    m = [t.double().cpu() for t in net.wide.momentum]
    w = [t.double().cpu() for t in net.wide.master]
    v0 = net.vectors[1]["scale"].double().cpu()
    for step in range(2):
        net.forward(x)
        net.scores(labels)
        net.backward(labels)
        norm, scale, clipped = ref.clip(net.gradients(), math.inf if max_norm is None else max_norm)
        dv = net.dvectors[1]["scale"].double().cpu()
        net.update(lr=0.02, mu=0.9)
        if max_norm is not None:
            assert float(net.norm) == pytest.approx(norm, rel=1e-6)
        first = len(net.blocks) + len(net.gates)
        for k in range(3):
            out = operators_ref.ortho_step(clipped[first + k].cpu(), m[k], 0.9, True, 5, w[k], 0.02 * math.sqrt(max(1.0, w[k].shape[1] / w[k].shape[2])))
            m[k], w[k] = out["momentum"], out["master"]
            assert float((net.wide.master[k].double().cpu() - w[k]).norm()) <= 1e-4 * float(w[k].norm()), k
            assert torch.equal(net.wide.weights[k], net.wide.master[k][0].to(net.wide.weights[k].dtype))
        v0 = v0 - 0.02 * scale * dv
        assert float((net.vectors[1]["scale"].double().cpu() - v0).abs().max()) <= 1e-6
    net.close()


def test_the_same_without_the_new_parts():
    """max_norm beyond the gradients' norm changes nothing in a network of the parts that were there before."""
    nets = [training.BlockNet(SHAPE, CLASSES, 1, "f32", GROUPS, max_norm=k) for k in (None, 1e9)]
    x, labels = training.synthetic(SHAPE[0], SHAPE, CLASSES, torch.float32, 4)
    for net in nets:
        for _ in range(2):
            net.forward(x)
            net.scores(labels)
            net.backward(labels)
            net.update()
    assert all(torch.equal(a, b) for d, e in zip(nets[0].blocks, nets[1].blocks) for a, b in zip(d.master, e.master))
    assert all(torch.equal(nets[0].vectors[1][k], nets[1].vectors[1][k]) for k in nets[0].vectors[1])
    for net in nets:
        net.close()
