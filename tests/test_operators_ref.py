"""The 64-bit definitions that the kernels are compared with: their gradients against central differences."""
import math

import pytest
import torch

import operators_ref as ref

# central differences in 64 bits with step h: truncation h^2 |f'''| / 6 ~ 1e-10 and rounding 2^-53 |f| / h ~ 1e-10 for
# values of order one
H, TOL = 1e-5, 1e-7


def _check(f, grads, tensors, gen):
    for name, t in tensors.items():
        d = torch.randn(t.shape, generator=gen, dtype=torch.float64)
        d /= d.norm()
        up, down = f(**{**tensors, name: t + H * d}), f(**{**tensors, name: t - H * d})
        got, want = float((grads[name] * d).sum()), float((up - down) / (2 * H))
        assert abs(got - want) <= TOL * max(1.0, abs(want)), (name, got, want)


@pytest.mark.parametrize("gate", [0, 1, 2])
@pytest.mark.parametrize("shape", [(2, 5, 3), (1, 1, 1), (3, 8, 1)])
@pytest.mark.parametrize("post,pre", [(True, True), (False, True), (True, False)])
def test_norm_gradients_against_differences(gate, shape, post, pre):
    if gate and not post:
        pytest.skip("a gate needs the block's output")
    gen = torch.Generator().manual_seed(3)
    rnd = lambda *s: torch.randn(*s, generator=gen, dtype=torch.float64)  # noqa: E731
    n, c, p = shape
    x, dy, du = rnd(*shape), rnd(*shape), rnd(*shape)
    t = {"x": x}
    if post:
        t |= {"z": rnd(*shape), "w_post": rnd(c), "scale": rnd(c)}
        if gate:
            t["g"] = rnd(*shape)
    if pre:
        t["w_pre"] = rnd(c)

    def loss(x, z=None, g=None, w_post=None, scale=None, w_pre=None):
        y, u = ref.norm_forward(x, z, g, w_post, scale, w_pre, gate, 0.1)
        return (y * dy).sum() + ((u * du).sum() if u is not None else 0)

    y, _ = ref.norm_forward(x, t.get("z"), t.get("g"), t.get("w_post"), t.get("scale"), t.get("w_pre"), gate, 0.1)
    got = ref.norm_backward(y, t.get("z"), t.get("g"), t.get("w_post"), t.get("scale"), t.get("w_pre"), gate, 0.1, dy, du if pre else None)
    names = {"x": "dx", "z": "dz", "g": "dgate", "w_post": "dw_post", "scale": "dscale", "w_pre": "dw_pre"}
    grads = {k: got.get(names[k], dy) for k in t}      # without PRE the gradient of x is dy itself
    _check(loss, grads, t, gen)


@pytest.mark.parametrize("classes,masked,it", [(1, False, 1.0), (7, False, 0.7), (7, True, 1.3), (40, True, 1.0)])
def test_logprob_gradients_against_differences(classes, masked, it):
    gen = torch.Generator().manual_seed(5)
    rows = 4
    logits = torch.randn(rows, classes, generator=gen, dtype=torch.float64) * 2
    tokens = torch.randint(0, classes, (rows,), generator=gen)
    tokens[1] = -1
    mask = None
    if masked:
        mask = torch.rand(rows, classes, generator=gen) < 0.6
        mask[torch.arange(rows), tokens.clamp(min=0)] = True
        mask[3] = False
    dlp, dent = torch.randn(rows, generator=gen, dtype=torch.float64), torch.randn(rows, generator=gen, dtype=torch.float64)

    def loss(logits):
        o = ref.logprob_forward(logits, it, mask, tokens, 0)
        alive = o["logprob"] > -math.inf
        return (o["logprob"][alive] * dlp[alive]).sum() + (o["entropy"] * dent).sum()

    grad = ref.logprob_backward(logits, it, mask, tokens, dlp, dent)
    assert grad.abs().max() < 100
    _check(loss, {"logits": grad}, {"logits": logits}, gen)


def test_newton_schulz_brings_the_singular_values_near_one():
    gen = torch.Generator().manual_seed(7)
    for shape in [(8, 8), (5, 40), (40, 5)]:
        s = torch.linalg.svdvals(ref.newton_schulz(torch.randn(*shape, generator=gen, dtype=torch.float64), 6))
        assert 0.5 < float(s.min()) and float(s.max()) < 1.3
