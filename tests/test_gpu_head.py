"""Log probabilities from features and the head's weight, and their gradients, against the definition in 64 bits, element by element."""
import math

import pytest
import torch

import more_operators_ref as ref
from paper_2304_07741_amd import binding as B
from paper_2304_07741_amd import harness

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
# rows, features, classes: single ones, sizes that no tile, vector or wave divides, the borders of the path for few rows (16, 32), one tile and
# one more than it, sums cut into parts
SHAPES = [(1, 1, 1), (1, 8, 2), (2, 3, 5), (4, 2048, 500), (16, 40, 33), (17, 100, 1000), (32, 65, 257), (33, 40, 24), (64, 64, 100), (129, 72, 129), (256, 512, 1000),
          (300, 1000, 131), (9000, 16, 40), (700, 33, 3001)]


def _case(rows, features, classes, dtype, seed, masked, std=2.5):
    gen = torch.Generator().manual_seed(seed)
    dt = TYPES[dtype]
    x = torch.randn(rows, features, generator=gen).to(dt)
    w = (torch.randn(classes, features, generator=gen) * (std / features ** 0.5)).to(dt)
    tokens = torch.randint(0, classes, (rows,), generator=gen)
    mask = None
    if masked:
        mask = torch.rand(classes, generator=gen) < 0.6
        mask[int(tokens[0])] = True
    if rows > 8:
        tokens[1], tokens[2], tokens[3] = -1, classes, -(1 << 40)     # positions without a target
        tokens[4] = (x[4].float() @ w.float().T).argmax()
    return x.cuda(), w.cuda(), tokens.cuda(), None if mask is None else mask.cuda(), torch.randn(rows, generator=gen).cuda(), torch.randn(rows, generator=gen).cuda()


def _run(x, w, tokens, mask, dlp, dent, dtype, it=1.0, flags=0):
    r = harness.HeadRunner(x.shape[0], x.shape[1], w.shape[0], dtype, flags=flags)
    for t in [*r.out.values(), *r.grads.values()]:
        t.fill_(float("nan"))
    r.ws.fill_(0xFF)
    out = {k: v.clone() for k, v in r.forward(x, w, tokens, mask=mask, inv_temperature=it).items()}
    if not flags:
        out |= {k: v.clone() for k, v in r.backward(x, w, tokens, dlp, dent, mask=mask, inv_temperature=it).items()}
    torch.cuda.synchronize()
    r.close()
    return out


def _compare(got, val, bound, f32, what):
    for name, v in val.items():
        g = got[name].double()
        assert g.shape == v.shape, (what, name)
        fine = torch.isfinite(v)
        assert torch.equal(g[~fine], v[~fine]) and bool(torch.isfinite(g[fine]).all()), (what, name)
        over = ((g - v).abs() - bound[name] - 1e-37)[fine]
        assert over.numel() == 0 or float(over.max()) <= 0, (what, name, float((g - v)[fine].abs().max()), int((over > 0).sum()))
        rel = float((g - v)[fine].norm() / v[fine].norm().clamp_min(1e-30))
        if name in ("dx", "dweight") and not f32 and got["logprob"].numel() >= 1000 and val["dweight"].shape[0] >= 1000:
            # two roundings to the type, uniform within half a step each (rms half / 3^(1/2)), of gradients of which 1000 at least, one a row, weigh alike
            assert rel <= 2.0 ** -8, (what, name, rel)


def _check(case, dtype, it, what, dlp=True, dent=True):
    x, w, tokens, mask, a, b = case
    a, b = a if dlp else None, b if dent else None
    val, bound = ref.head(x.double(), w.double(), tokens, it, mask, None if a is None else a.double(), None if b is None else b.double(), f32=dtype == "f32")
    _compare(_run(x, w, tokens, mask, a, b, dtype, it), val, bound, dtype == "f32", what)


@pytest.mark.parametrize("masked", [False, True], ids=["all", "masked"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_against_the_definition(shape, dtype, masked):
    _check(_case(*shape, dtype, 3 + sum(shape), masked), dtype, 1.0 if masked else 0.7, (shape, dtype, masked))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(40000, 40, 4000), (3000, 64, 6100), (100000, 24, 700), (250000, 24, 700)], ids=str)
def test_several_pieces_and_large_tiles(shape, dtype):
    if dtype == "f32" and shape[0] >= 100000:
        pytest.skip("the first shape has pieces of fp32 plans")
    case = _case(*shape, dtype, 5, shape[0] == 3000)
    plan = harness.HeadRunner(*shape, dtype)
    assert (plan.info.pieces > 1) == (shape[0] * shape[2] * (6 if dtype == "f32" else 2) > 288 << 20)
    plan.close()
    _check(case, dtype, 1.0, (shape, dtype))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(17, 33, 16385), (32, 72, 17001)], ids=str)
def test_few_rows_of_many_classes(shape, dtype):
    _check(_case(*shape, dtype, 6, True), dtype, 1.0, (shape, dtype))


def test_logits_of_some_pieces_are_left_for_backward():
    """More than a GiB of logits: those of the first pieces are read again, the others computed again."""
    shape = (70000, 200, 4100)
    case = _case(*shape, "f32", 9, True)
    plan = harness.HeadRunner(*shape, "f32")
    assert plan.info.pieces > 8 and 1 << 30 < 4 * shape[0] * shape[2]
    plan.close()
    _check(case, "f32", 0.8, shape)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_long_sums(dtype):
    _check(_case(1001, 1993, 8101, dtype, 8, True), dtype, 1.0, dtype)


@pytest.mark.parametrize("dlp,dent", [(True, False), (False, True), (False, False)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gradients_that_are_not_given(dtype, dlp, dent):
    _check(_case(70, 40, 300, dtype, 6, True), dtype, 1.5, (dtype, dlp, dent), dlp, dent)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [5, 60])
def test_nothing_left(dtype, rows):
    """All classes masked: log probability -inf (0 without a token), entropy 0, gradients of zeros."""
    x, w, tokens, _, a, b = _case(rows, 24, 90, dtype, 2, False)
    tokens[0] = -1
    got = _run(x, w, tokens, torch.zeros(90, dtype=torch.bool, device="cuda"), a, b, dtype)
    given = (tokens >= 0) & (tokens < 90)
    assert torch.equal(got["logprob"], torch.where(given, -math.inf, 0.0))
    assert not got["entropy"].any() and not got["dx"].any() and not got["dweight"].any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [9, 150])
def test_what_is_hidden_is_not_looked_at(dtype, rows):
    """NaN and infinities in the weight of masked classes and in the features of rows without a target change nothing."""
    x, w, tokens, mask, a, _ = _case(rows, 40, 300, dtype, 4, True)
    want = _run(x, w, tokens, mask, a, None, dtype)
    w2, x2 = w.clone(), x.clone()
    hidden = (~mask).nonzero()[:, 0]
    w2[hidden[0]], w2[hidden[1], 3], w2[hidden[2]] = math.nan, math.inf, -math.inf
    got = _run(x2, w2, tokens, mask, a, None, dtype)
    assert all(torch.equal(got[k], want[k]) for k in want)
    x2[1], x2[2, 5] = math.nan, math.inf          # tokens[1] and tokens[2] are no classes
    got = _run(x2, w2, tokens, mask, a, None, dtype)
    assert torch.equal(got["dx"], want["dx"]) and torch.equal(got["dweight"], want["dweight"]) and torch.equal(got["logprob"], want["logprob"])
    assert not want["dx"][1:4].any() and not want["dweight"][~mask].any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [7, 100])
def test_logits_that_are_not_finite(dtype, rows):
    x, w, tokens, _, a, b = _case(rows, 16, 200, dtype, 8, False)
    tokens = torch.randint(0, 200, (rows,), device="cuda")
    x[3, 2] = math.nan
    got = _run(x, w, tokens, None, a, b, dtype)
    bad = torch.zeros(rows, dtype=torch.bool, device="cuda")
    bad[3] = True
    for name in ("logprob", "entropy"):
        assert torch.equal(torch.isnan(got[name]), bad)
    assert torch.equal(torch.isnan(got["dx"]).any(1), bad) and bool(torch.isnan(got["dweight"]).all())
    val, _ = ref.head(x.double()[~bad], w.double(), tokens[~bad], grads=False)
    assert float((got["logprob"][~bad].double() - val["logprob"]).abs().max()) < 1e-4


@pytest.mark.parametrize("it", [1e-30, 1e-3, 50.0, 3.4e38])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_temperatures(dtype, it):
    """From distributions that are flat to those that one class has."""
    x, w, tokens, mask, a, b = _case(60, 32, 500, dtype, 10, False)
    if it <= 50:
        _check((x, w, tokens, mask, a, b), dtype, it, (dtype, it))
    else:
        # logits in steps of 2^-8: differences are zero or beyond every exponential
        x, w = (x * 4).round().clamp(-8, 8) / 4, (w * 4).round() / 4
        tokens[:] = (x.float() @ w.float().T).argmax(1)
        got = _run(x, w, tokens, mask, torch.zeros_like(a), None, dtype, it)
        same = ((x.double() @ w.double().T) == (x.double() @ w.double().T).amax(1, keepdim=True)).sum(1)
        assert float((got["logprob"].double() + torch.log(same.double())).abs().max()) <= 1e-6
        assert float((got["entropy"].double() - torch.log(same.double())).abs().max()) <= 1e-6


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [4, 32, 200])
def test_the_same_as_from_logits(dtype, rows):
    """canvas_logprob on the logits that fp32 gives: the same conventions, the same values."""
    x, w, tokens, mask, a, b = _case(rows, 64, 777, dtype, 12, True)
    tokens[0] = -1
    tokens[1] = int((~mask).nonzero()[0, 0])
    got = _run(x, w, tokens, mask, a, b, dtype, 0.8)
    logits = (x.double() @ w.double().T).float().contiguous()
    r = harness.LogprobRunner(rows, 777, "f32")
    want = r.forward(logits, tokens, mask=mask, inv_temperature=0.8)
    for name in ("logprob", "entropy"):
        g, v = got[name], want[name]
        assert torch.equal(torch.isinf(g), torch.isinf(v))
        fine = torch.isfinite(v)
        # (logits here are sums of 64 products in fp32: 66 u times the sum of their magnitudes, which is below 64 4 2.5 / 8 4)
        assert float((g - v)[fine].abs().max()) <= 4e-4
    r.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 1, 1), (5, 333, 70), (32, 64, 1000), (40, 33, 300), (300, 512, 200)], ids=str)
def test_inference_plans_give_the_same(shape, dtype):
    case = _case(*shape, dtype, 13, True)
    full, infer = _run(*case, dtype), _run(*case, dtype, flags=B.CANVAS_OPT_INFERENCE)
    assert torch.equal(full["logprob"], infer["logprob"]) and torch.equal(full["entropy"], infer["entropy"])


def test_gradients_against_differences():
    """sum(logprob a + entropy b) from the kernels themselves in fp32: central differences along random directions."""
    x, w, tokens, mask, a, b = _case(60, 24, 130, "f32", 14, True)
    r = harness.HeadRunner(60, 24, 130, "f32")
    ok = torch.isfinite(r.forward(x, w, tokens, mask=mask)["logprob"])
    a = torch.where(ok, a, torch.zeros_like(a))       # (the log probability of a masked token is -inf wherever one goes)
    g = {k: v.clone() for k, v in r.backward(x, w, tokens, a, b, mask=mask).items()}
    gen = torch.Generator().manual_seed(1)
    for name, at in (("dx", 0), ("dweight", 1)):
        v = torch.randn((x, w)[at].shape, generator=gen).cuda()
        loss = []
        for s in (1, -1):
            moved = [x, w]
            moved[at] = moved[at] + s * 2.0 ** -9 * v
            o = r.forward(*moved, tokens, mask=mask)
            loss.append(float((o["logprob"].double() * a.double())[ok].sum() + (o["entropy"].double() * b.double()).sum()))
        want, got = (loss[0] - loss[1]) / 2.0 ** -8, float((g[name].double() * v.double()).sum())
        assert abs(want - got) <= 2e-3 * float(g[name].double().norm() * v.double().norm()), (name, want, got)
    r.close()


@pytest.mark.parametrize("rows", [3, 20, 40, 1500])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gradients_of_cold_distributions_add_up_to_nothing(dtype, rows):
    # The gradients of a row's logits add up to zero, which a column of ones in W shows in dx, however much the temperature multiplies the rounding of the logits:
    # forward and backward have to mean the same logits.  Per unit of |g| it: 500 terms and their sum of e^x, fp32, each off by at most (500 + 90 * 3 + 8) 2^-24
    # (the sum, three roundings of an argument that is 90 at most, or 126 in powers of two, the rest), once for p and once for the sum that dx is: 2^-12.
    # bf16: dlogit's rounding, half a step of numbers that add up to 2 |g| it in all, 2^-7, and dx's own.
    it, classes, features = 1e6, 500, 136
    gen = torch.Generator().manual_seed(rows)
    dt = TYPES[dtype]
    x = torch.randn(rows, features, generator=gen).to(dt).cuda()
    w = torch.randn(classes, features, generator=gen).to(dt)
    x[:, 0], w[:, 0] = 0, 1
    tokens = torch.randint(0, classes, (rows,), generator=gen).cuda()
    g = torch.randn(rows, generator=gen).cuda()
    out = _run(x, w.cuda(), tokens, None, g, None, dtype, it=it)
    left = out["dx"][:, 0].double().abs() / (g.double().abs() * it)
    assert float(left.max()) <= (2.0 ** -12 if dtype == "f32" else 2.0 ** -7 * (1 + 2.0 ** -8) + 2.0 ** -12), left.max()
