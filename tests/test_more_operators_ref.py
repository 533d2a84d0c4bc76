"""The definitions in 64 bits that the kernels are compared with, against differences of themselves and against torch's own gradients (CPU)."""
import pytest
import torch

import more_operators_ref as ref


@pytest.mark.parametrize("kind", [0, 1, 2])
def test_gated_gradients(kind):
    gen = torch.Generator().manual_seed(kind)
    x, wg, wu, dy = (torch.randn(*s, generator=gen, dtype=torch.float64) for s in ((5, 4), (7, 4), (7, 4), (5, 7)))
    leaves = [v.clone().requires_grad_() for v in (x, wg, wu)]
    g, u = leaves[0] @ leaves[1].T, leaves[0] @ leaves[2].T
    a = {0: torch.sigmoid, 1: torch.nn.functional.silu, 2: torch.nn.functional.gelu}[kind](g)
    grads = torch.autograd.grad((a * u * dy).sum(), leaves)
    val, bound = ref.gated(kind, x, wg, wu, dy)
    assert torch.allclose(val["y"], (a * u).detach(), rtol=1e-12, atol=1e-12)
    for name, v in zip(("dx", "dw_gate", "dw_up"), grads):
        assert torch.allclose(val[name], v, rtol=1e-11, atol=1e-11)
        assert bool((bound[name] > 0).all()) and float((bound[name] / (1 + v.abs())).max()) < 1e-3


@pytest.mark.parametrize("masked", [False, True])
def test_head_gradients(masked):
    gen = torch.Generator().manual_seed(3)
    x, w = torch.randn(6, 4, generator=gen, dtype=torch.float64), torch.randn(9, 4, generator=gen, dtype=torch.float64)
    tokens = torch.tensor([0, 3, 8, -1, 9, 5])
    mask = None if not masked else torch.tensor([1, 0, 1, 1, 1, 1, 0, 1, 1]).bool()
    a, b = torch.randn(6, generator=gen, dtype=torch.float64), torch.randn(6, generator=gen, dtype=torch.float64)
    lx, lw = x.clone().requires_grad_(), w.clone().requires_grad_()
    z = lx @ lw.T * 0.6
    if masked:
        z = z[:, mask]
    logp = torch.log_softmax(z, 1)
    place = {c: k for k, c in enumerate(range(9) if mask is None else mask.nonzero()[:, 0].tolist())}
    loss = sum(a[t] * logp[t, place[int(c)]] for t, c in enumerate(tokens) if int(c) in place) - (b * (logp.exp() * logp).sum(1)).sum()
    gx, gw = torch.autograd.grad(loss, (lx, lw))
    val, bound = ref.head(x, w, tokens, 0.6, mask, a, b)
    assert torch.allclose(val["dx"], gx, rtol=1e-10, atol=1e-12) and torch.allclose(val["dweight"], gw, rtol=1e-10, atol=1e-12)
    assert float(val["logprob"][3]) == 0 and float(val["logprob"][4]) == 0
    assert torch.allclose(val["entropy"], -(logp.exp() * logp).sum(1).detach(), rtol=1e-12)
    assert float(bound["dx"].max()) < 1e-3


def test_clip():
    g = [torch.tensor([3.0]), torch.tensor([0.0, 4.0])]
    norm, scale, out = ref.clip(g, 1.0)
    assert norm == 5 and scale == 0.2 and torch.allclose(out[1], torch.tensor([0.0, 0.8], dtype=torch.float64))
    assert ref.clip(g, 10.0)[1] == 1 and ref.clip([torch.zeros(3)], 1.0)[1] == 1
