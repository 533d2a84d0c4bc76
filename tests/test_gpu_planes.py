"""fp32 plans of gated pairs and heads: single products, and errors over all results that tell three planes of an operand from two (test_planes_ref.py)."""
import pytest
import torch

import more_operators_ref as ref
import planes_ref
from paper_2304_07741_amd import binding as B
from paper_2304_07741_amd import harness
from planes_ref import U

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("power", [0, -98])
def test_single_products(power):
    # One feature and gates of zero: y = x w / 2.  Off by what the six products leave out, their sum, the sigmoid of zero (two roundings) and the product with it:
    # (1 + 1 + 2 + 1) u, and a hundredth for the small products' sum.  In the mean by nothing: 5000 x and 64 w of both signs, less than u / 4 each, w's eighth of that left.
    rows, width = 5000, 64
    gen = torch.Generator().manual_seed(1)
    x, w = torch.randn(rows, 1, generator=gen), torch.randn(width, 1, generator=gen)
    x[:4, 0] = torch.tensor([1.0078124, -1.0078124, 1.9999999, 1.0039061])
    w[:4, 0] = x[:4, 0]
    x, w = torch.where(x.abs() < 0.25, x + torch.copysign(torch.full_like(x, 0.25), x), x) * 2.0 ** power, w * 2.0 ** -power   # (operands from 2^-100 on)
    r = harness.GatedRunner(rows, 1, width, "f32", B.CANVAS_GATED_SIGMOID, flags=B.CANVAS_OPT_INFERENCE)
    assert r.info.n_launches_fwd == 2                     # copies in planes, and tiles
    x, w = x.cuda(), w.cuda()
    y = r.forward(x, torch.zeros_like(w), w)["y"].double()
    want = 0.5 * x.double() @ w.double().T
    rel = (y - want) / want
    assert float(rel.abs().max()) <= 5.1 * U, float(rel.abs().max()) / U
    assert abs(float(rel.mean())) <= 0.25 * U, float(rel.mean()) / U
    r.close()


def test_results_of_gated_pairs():
    # silu: 0.65 of a gate's error goes to act, 0.6 in the mean square itself, so g and u make y off by 2.1 times theirs at most, act by a few u
    rows, features, width = 5000, 100, 200
    gen = torch.Generator().manual_seed(2)
    x, wg, wu = (torch.randn(s, features, generator=gen) for s in (rows, width, width))
    t = [x.cuda(), (wg / 10).cuda(), (wu / 10).cuda()]
    r = harness.GatedRunner(rows, features, width, "f32", flags=B.CANVAS_OPT_INFERENCE)
    assert r.info.n_launches_fwd == 2
    y = r.forward(*t)["y"]
    val, _ = ref.gated(1, *(v.double() for v in t))
    got = planes_ref.off(y, val["y"])
    print("y", got, flush=True)
    assert got <= 2.1 * planes_ref.product_off(features) + 8 * U <= planes_ref.TWO
    r.close()


@pytest.mark.parametrize("rows", [100, 200])
def test_gradients_of_gated_pairs(rows):
    # dg and du: 2.1 times g's and u's error (as above; silu'' is below silu' in the mean), a few u; then their own product
    features, width = 60, 150
    gen = torch.Generator().manual_seed(3)
    x, wg, wu, dy = (torch.randn(*s, generator=gen) for s in ((rows, features), (width, features), (width, features), (rows, width)))
    t = [x.cuda(), (wg / features ** 0.5).cuda(), (wu / features ** 0.5).cuda(), dy.cuda()]
    r = harness.GatedRunner(rows, features, width, "f32")
    r.forward(*t[:3])
    got = r.backward(*t)
    val, _ = ref.gated(1, *(v.double() for v in t))
    before = 2.1 * planes_ref.product_off(features) + 12 * U
    for name, n in (("dx", 2 * width), ("dw_gate", rows), ("dw_up", rows)):
        o = planes_ref.off(got[name], val[name])
        print(name, o, flush=True)
        assert o <= before + planes_ref.product_off(n) <= planes_ref.TWO, name
    r.close()


def test_log_probabilities():
    # logits of size 8:   Off by the token's logit and the mean of the others', each product_off of 8, and by
    # roundings of numbers as large as the log probability: the difference from the largest, its exponential's argument, the sum's logarithm and the last difference
    rows, features, classes = 5000, 100, 300
    gen = torch.Generator().manual_seed(5)
    x, w = torch.randn(rows, features, generator=gen).cuda(), (torch.randn(classes, features, generator=gen) * 0.8).cuda()
    tokens = torch.randint(0, classes, (rows,), generator=gen).cuda()
    r = harness.HeadRunner(rows, features, classes, "f32", flags=B.CANVAS_OPT_INFERENCE)
    assert r.info.n_launches_fwd == 3
    got = r.forward(x, w, tokens)["logprob"].double()
    val, _ = ref.head(x.double(), w.double(), tokens, grads=False)
    size = float(val["logprob"].norm()) / rows ** 0.5
    o = float((got - val["logprob"]).norm()) / rows ** 0.5
    print("logprob", o, "of", size, flush=True)
    assert o <= 2 * 8 * planes_ref.product_off(features) + 4 * size * U <= 8 * planes_ref.TWO
    r.close()


@pytest.mark.parametrize("rows", [60, 200])
def test_gradients_of_heads(rows):
    # logits of size 1: a dlogit is off by p times twice their error, and by a few u of itself and of g; then its own product
    features, classes = 40, 300
    gen = torch.Generator().manual_seed(6)
    x, w = torch.randn(rows, features, generator=gen).cuda(), (torch.randn(classes, features, generator=gen) / features ** 0.5).cuda()
    tokens, g, h = torch.randint(0, classes, (rows,), generator=gen).cuda(), torch.randn(rows, generator=gen).cuda(), torch.randn(rows, generator=gen).cuda()
    r = harness.HeadRunner(rows, features, classes, "f32")
    r.forward(x, w, tokens)
    got = r.backward(x, w, tokens, g, h)
    val, _ = ref.head(x.double(), w.double(), tokens, 1.0, None, g.double(), h.double())
    before = 2 * planes_ref.product_off(features) + 12 * U
    for name, n in (("dx", classes), ("dweight", rows)):
        o = planes_ref.off(got[name], val[name])
        print(name, o, flush=True)
        assert o <= before + planes_ref.product_off(n) <= planes_ref.TWO, name
    r.close()
