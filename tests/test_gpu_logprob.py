"""Log probabilities of given tokens, entropy, top alternatives and their gradient against the definition in 64 bits."""
import math

import numpy as np
import pytest
import torch

import operators_ref as ref
from paper_2304_07741_amd import binding as B
from paper_2304_07741_amd import harness

pytestmark = pytest.mark.gpu

# rows, classes, elements between the rows: one row and one class, rows shorter than a wavefront, odd lengths at odd
# addresses, vocabularies that one workgroup holds and that it does not
SHAPES = [(1, 1, 0), (3, 2, 0), (5, 7, 1), (4, 64, 0), (300, 33, 0), (17, 1000, 0), (3, 1023, 3), (2, 8192, 8), (600, 2049, 0), (4, 50021, 2), (1, 131072, 0),
          (2, 200003, 1), (1, 1000001, 0)]


def _case(rows, classes, pad, dtype, masked, seed, it):
    gen = torch.Generator().manual_seed(seed)
    dt = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    wide = (torch.randn(rows, classes + pad, generator=gen) * 3).to(dt)
    tokens = torch.randint(0, classes, (rows,), generator=gen)
    tokens[rows // 2] = wide[rows // 2, :classes].float().argmax()
    if rows > 2:
        tokens[1], tokens[2] = -1, classes      # positions without a target
    mask = None
    if masked:
        mask = torch.rand(rows, classes, generator=gen) < 0.5
        if rows > 4:
            mask[4] = False                     # nothing left
    return wide, tokens, mask, it, torch.randn(rows, generator=gen), torch.randn(rows, generator=gen)


def _run(wide, classes, dtype, tokens, mask, it, dlp, dent, top, in_place=False):
    rows = wide.shape[0]
    r = harness.LogprobRunner(rows, classes, dtype, top_k=top)
    dev = wide.cuda()
    logits = dev[:, :classes]
    for t in [*r.out.values(), *r.grads.values()]:
        t.fill_(float("nan") if t.is_floating_point() else -7)
    r.ws.fill_(0xFF)
    m = None if mask is None else mask.cuda()
    out = {k: v.clone() for k, v in r.forward(logits, tokens.cuda(), mask=m, inv_temperature=it).items()}
    d1, d2 = (None if t is None else t.cuda() for t in (dlp, dent))
    if in_place:
        B.canvas_logprob_backward(r.handle, logits, dev.shape[1], it, m, 0 if m is None else classes, tokens.cuda(), d1, d2, logits, dev.shape[1], r.ws)
        out["dlogits"] = logits.clone()
        assert torch.equal(dev[:, classes:].cpu(), wide[:, classes:])          # nothing between the rows is written
    else:
        out |= r.backward(logits, tokens.cuda(), d1, d2, mask=m, inv_temperature=it)
    torch.cuda.synchronize()
    res = {k: v.cpu() for k, v in out.items()}
    r.close()
    return res


def _same(got, want, rel, scale, what):
    got, want = got.double().numpy(), want.double().numpy()
    assert got.shape == want.shape
    assert (np.isnan(got) == np.isnan(want)).all() and (np.isinf(got) == np.isinf(want)).all(), what
    fin = np.isfinite(want)
    bad = np.abs(got[fin] - want[fin]) > rel * np.maximum(np.abs(want[fin]), scale)
    assert not bad.any(), (what, np.abs(got[fin] - want[fin]).max())


# fp32: a log probability is a difference of numbers below 64 in magnitude (2^-24 each: 4e-6 absolute) and the logarithm of a
# sum of up to 10^6 terms whose partial sums are rounded some 20 times (2e-6); gradients carry the same relative error.  bf16
# gradients are rounded once: 2^-9.
ABS = 1e-5


def _check(got, want, grad, dtype, dlp, dent, classes, it):
    _same(got["logprob"], want["logprob"], ABS, 1.0, "logprob")
    _same(got["entropy"], want["entropy"], ABS, 1.0, "entropy")
    if "top_index" in got:
        assert torch.equal(got["top_index"].to(torch.int64), want["top_index"])
        _same(got["top_logprob"], want["top_logprob"], ABS, 1.0, "top_logprob")
    if grad is not None:
        # elements far below the row's largest are held to the absolute bound of the largest one
        size = float(grad[torch.isfinite(grad)].abs().max()) if torch.isfinite(grad).any() else 1.0
        rel = ABS if dtype == "f32" else 2.0 ** -8
        _same(got["dlogits"], grad, rel, max(size, 1e-30) * (1.0 if dtype == "f32" else 1e-3), "dlogits")


@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_forward_and_backward(shape, dtype, masked):
    rows, classes, pad = shape
    top = {0: 5, 1: 64, 2: 1}[classes % 3]
    wide, tokens, mask, it, dlp, dent = _case(rows, classes, pad, dtype, masked, sum(shape), 0.8 if masked else 1.0)
    logits = wide[:, :classes].double()
    want = ref.logprob_forward(logits, it, mask, tokens, top)
    grad = ref.logprob_backward(logits, it, mask, tokens, dlp.double(), dent.double())
    got = _run(wide, classes, dtype, tokens, mask, it, dlp, dent, top)
    _check(got, want, grad, dtype, dlp, dent, classes, it)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("masked", [False, True])
def test_gradient_in_the_place_of_the_logits(dtype, masked):
    for rows, classes, pad in [(3, 1023, 3), (6, 4096, 0), (2, 70001, 5)]:
        wide, tokens, mask, it, dlp, dent = _case(rows, classes, pad, dtype, masked, 8, 1.5)
        a = _run(wide, classes, dtype, tokens, mask, it, dlp, dent, 0)
        b = _run(wide, classes, dtype, tokens, mask, it, dlp, dent, 0, in_place=True)
        for k in a:
            assert torch.equal(a[k].view(torch.int16 if a[k].dtype == torch.bfloat16 else torch.int32), b[k].view(torch.int16 if b[k].dtype == torch.bfloat16 else torch.int32)), k


@pytest.mark.parametrize("classes", [40, 1000, 30000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_ties_go_to_the_lowest_index(dtype, classes):
    gen = torch.Generator().manual_seed(1)
    wide = torch.randint(-2, 3, (6, classes), generator=gen).to({"f32": torch.float32, "bf16": torch.bfloat16}[dtype])
    wide[0] = 0.25                                          # all the same
    wide[1] = torch.arange(classes).flip(0).to(wide.dtype)  # descending
    wide[2] = torch.arange(classes).to(wide.dtype)          # ascending
    wide[3, :-70] = -1
    wide[3, -70:] = 5                                       # the best ones side by side at the end
    wide[4] = -0.0
    wide[4, 5::2] = 0.0                                     # zeros of both signs
    tokens = torch.zeros(6, dtype=torch.int64)
    want = ref.logprob_forward(wide.double(), 1.0, None, tokens, 64 if classes > 64 else 33)
    got = _run(wide, classes, dtype, tokens, None, 1.0, None, None, 64 if classes > 64 else 33)
    assert torch.equal(got["top_index"].to(torch.int64), want["top_index"])
    _same(got["top_logprob"], want["top_logprob"], ABS, 1.0, "top")
    assert (got["dlogits"] == 0).all()                      # no gradient came in


def _strange(dtype, classes):
    dt = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    gen = torch.Generator().manual_seed(2)
    w = (torch.randn(9, classes, generator=gen) * 2).to(dt)
    low = torch.finfo(dt).min
    w[0] = -math.inf                  # a row that a mask of infinities has emptied
    w[1, 3:] = -math.inf              # three classes left
    w[2] = low                        # all at the type's lowest value: uniform
    w[3, 1::2] = low                  # a mask of lowest values
    w[4, 7] = math.nan                # one NaN
    w[5, 9] = math.inf                # one infinity
    w[6] = math.nan                   # all NaN
    w[7, 2] = torch.finfo(dt).max     # one class takes all
    w[8, ::3] = -math.inf
    return w


@pytest.mark.parametrize("it", [1.0, 1.5])
@pytest.mark.parametrize("classes", [50, 5000, 140001])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_infinities_lowest_values_and_nan(dtype, classes, it):
    w = _strange(dtype, classes)
    tokens = torch.tensor([2, 1, 4, 0, 3, 9, 1, 2, 0])
    dlp, dent = torch.linspace(-1, 1, 9), torch.linspace(0.5, -0.5, 9)
    want = ref.logprob_forward(w.double(), it, None, tokens, 5)
    got = _run(w, classes, dtype, tokens, None, it, dlp, dent, 5)
    # (a class 10^38 below the largest has a log probability of that size: relative, and its overflow is -inf)
    fin = [1, 2, 3, 8]
    grad = ref.logprob_backward(w.double(), it, None, tokens, dlp.double(), dent.double())
    _same(got["logprob"][fin], want["logprob"][fin], ABS, 1.0, "logprob")
    _same(got["entropy"], want["entropy"], ABS, 1.0, "entropy")
    assert torch.equal(got["top_index"].to(torch.int64), want["top_index"])
    assert float(got["logprob"][0]) == -math.inf and (got["top_index"][0] == -1).all() and (got["dlogits"][0] == 0).all()
    assert float(got["logprob"][7]) == 0.0
    for r in (4, 5, 6):
        assert math.isnan(float(got["logprob"][r])) and torch.isnan(got["dlogits"][r].float()).all(), r
    rel = ABS if dtype == "f32" else 2.0 ** -8
    for r in (1, 2, 3, 7, 8):
        _same(got["dlogits"][r], grad[r], rel, float(grad[r].abs().max()) * (1.0 if dtype == "f32" else 1e-3) + 1e-30, f"dlogits {r}")


@pytest.mark.parametrize("classes", [50, 5000, 140001])
def test_what_a_mask_hides_is_not_looked_at(classes):
    """The same outputs whether masked logits are zeros, NaN or infinities; the gradient there is zero."""
    wide, tokens, mask, it, dlp, dent = _case(6, classes, 0, "f32", True, 3, 1.0)
    mask[torch.tensor([0, 3, 5]), tokens[torch.tensor([0, 3, 5])]] = True
    runs = []
    for v in (0.0, math.nan, math.inf, -math.inf):
        w = torch.where(mask, wide, torch.full((), v))
        runs.append(_run(w, classes, "f32", tokens, mask, it, dlp, dent, 3))
    for k in runs[0]:
        for r in runs[1:]:
            assert torch.equal(runs[0][k], r[k]), k
    assert (runs[0]["dlogits"][~mask] == 0).all() and (runs[0]["dlogits"][4] == 0).all()
    assert float(runs[0]["logprob"][4]) == -math.inf and float(runs[0]["entropy"][4]) == 0.0


def test_one_mask_for_all_rows_and_no_token():
    wide, tokens, mask, it, dlp, dent = _case(5, 700, 4, "bf16", True, 6, 0.5)
    tokens = tokens.clamp(0, 699)
    one = mask[0].clone()
    rows = one[None].expand(5, -1).contiguous()
    r = harness.LogprobRunner(5, 700, "bf16", top_k=3)
    logits = wide.cuda()[:, :700]
    outs = []
    for m in (one.cuda(), rows.cuda()):
        o = {k: v.clone() for k, v in r.forward(logits, tokens.cuda(), mask=m, inv_temperature=it).items()}
        o |= {k: v.clone() for k, v in r.backward(logits, tokens.cuda(), dlp.cuda(), dent.cuda(), mask=m, inv_temperature=it).items()}
        outs.append(o)
    for k in outs[0]:
        assert torch.equal(outs[0][k], outs[1][k]), k
    # entropy and alternatives without tokens
    ent = torch.full((5,), math.nan, device="cuda")
    top, idx = torch.empty(5, 3, device="cuda"), torch.empty(5, 3, dtype=torch.int32, device="cuda")
    B.canvas_logprob_forward(r.handle, logits, wide.shape[1], it, one.cuda(), 0, None, None, ent, top, idx, r.ws)
    assert torch.equal(ent, outs[0]["entropy"]) and torch.equal(idx, outs[0]["top_index"])
    r.close()


def test_two_runs_give_the_same_bits_on_another_stream():
    for rows, classes in [(3, 100000), (500, 3000)]:
        wide, tokens, mask, it, dlp, dent = _case(rows, classes, 0, "bf16", False, 13, 1.0)
        a = _run(wide, classes, "bf16", tokens, mask, it, dlp, dent, 10)
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            b = _run(wide, classes, "bf16", tokens, mask, it, dlp, dent, 10)
        for k in a:
            assert torch.equal(a[k], b[k]), k


def test_offsets_beyond_32_bits():
    """Rows that begin more than 2^32 bytes behind the first one: two rows of a wide buffer, every element NaN but theirs."""
    rows, classes, pitch = 3, 1000, (1 << 31) + 24
    buf = torch.empty(2 * pitch + classes, dtype=torch.bfloat16, device="cuda")
    gen = torch.Generator().manual_seed(3)
    vals = (torch.randn(rows, classes, generator=gen) * 2).bfloat16()
    for r in range(rows):
        buf[r * pitch : r * pitch + classes] = vals[r].cuda()
    logits = torch.as_strided(buf, (rows, classes), (pitch, 1))
    tokens = torch.tensor([1, 5, 999])
    r = harness.LogprobRunner(rows, classes, "bf16", top_k=4)
    out = {k: v.cpu() for k, v in r.forward(logits, tokens.cuda()).items()}
    want = ref.logprob_forward(vals.double(), 1.0, None, tokens, 4)
    _same(out["logprob"], want["logprob"], ABS, 1.0, "logprob")
    assert torch.equal(out["top_index"].to(torch.int64), want["top_index"])
    dlp = torch.ones(rows)
    B.canvas_logprob_backward(r.handle, logits, pitch, 1.0, None, 0, tokens.cuda(), dlp.cuda(), None, logits, pitch, r.ws)
    grad = ref.logprob_backward(vals.double(), 1.0, None, tokens, dlp.double(), None)
    _same(logits.cpu(), grad, 2.0 ** -8, 1e-3, "dlogits")
    r.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("top", [1, 5, 31, 32, 33])
@pytest.mark.parametrize("classes", [3, 31, 64, 700, 1024, 1025, 2048, 2049])
def test_alternatives_of_short_rows(classes, top, dtype):
    """Rows that a wave or a workgroup holds: ties, orders, infinities and NaN, with and without a mask."""
    top = min(top, classes)
    wide, tokens, mask, _, dlp, dent = _case(12, classes, 1, dtype, True, classes + top, 1.0)
    wide[0] = 0.25
    wide[1] = torch.arange(classes + 1).flip(0).to(wide.dtype)
    wide[2] = torch.arange(classes + 1).to(wide.dtype)
    wide[3] = (torch.arange(classes + 1) % 7).to(wide.dtype)
    wide[5, ::3] = -math.inf
    wide[6] = -math.inf
    wide[7, classes // 2] = math.nan
    wide[8, -2] = math.inf
    for m in (None, mask):
        want = ref.logprob_forward(wide[:, :classes].double(), 1.0, m, tokens, top)
        got = _run(wide, classes, dtype, tokens, m, 1.0, dlp, dent, top)
        grad = ref.logprob_backward(wide[:, :classes].double(), 1.0, m, tokens, dlp.double(), dent.double())
        _check(got, want, grad, dtype, dlp, dent, classes, 1.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("rows,classes,top", [(7, 3001, 20), (7, 4096, 32), (7, 4097, 32), (2050, 5003, 8), (2050, 4100, 0), (2050, 8193, 3)])
def test_rows_that_a_wave_takes_in_turns(rows, classes, top, masked, dtype):
    """All rows run; the definition is computed for the first and the last ones."""
    wide, tokens, mask, _, dlp, dent = _case(rows, classes, 1, dtype, masked, classes + top, 1.0)
    wide[0] = 0.25
    wide[1] = torch.arange(classes + 1).to(wide.dtype)
    some = sorted({*range(min(rows, 12)), *range(max(0, rows - 4), rows)})
    logits, part = wide[some, :classes].double(), None if mask is None else mask[some]
    want = ref.logprob_forward(logits, 1.0, part, tokens[some], top)
    grad = ref.logprob_backward(logits, 1.0, part, tokens[some], dlp[some].double(), dent[some].double())
    got = _run(wide, classes, dtype, tokens, mask, 1.0, dlp, dent, top)
    _check({k: v[some] for k, v in got.items()}, want, grad, dtype, dlp, dent, classes, 1.0)


@pytest.mark.parametrize("rows,classes", [(64, 1000), (3, 5003), (4, 131072), (2, 200003)])
def test_every_probability_in_the_gradient_to_a_few_units(rows, classes):
    """Logits whose differences fp32 holds: -dlogit / dlogprob is p, of which the exponential is good to a unit (2^-23), the sum's error is
    below 2e-7 (the threads' sums of some hundred terms, and the factor log2 e, 1.3e-8 of exponents around 8), and three roundings of 2^-24 follow:
    5e-7 in all, held to 8e-7 however small p is."""
    gen = torch.Generator().manual_seed(classes)
    logits = torch.round(torch.randn(rows, classes, generator=gen) * 2.5 * 256) / 256
    tokens = torch.full((rows,), -1)
    tokens[:] = torch.arange(rows) % classes
    got = _run(logits, classes, "f32", tokens, None, 1.0, torch.ones(rows), None, 0)["dlogits"].double()
    p = torch.softmax(logits.double(), 1)
    rest = torch.ones(rows, classes, dtype=torch.bool)
    rest[torch.arange(rows), tokens] = False
    off = (got + p).abs() / p
    assert float(p.min()) < 1e-7 and float(off[rest].max()) <= 8e-7
    # the token's own element is 1 - p
    own = got[torch.arange(rows), tokens] - (1 - p[torch.arange(rows), tokens])
    assert float(own.abs().max()) <= 2e-7


@pytest.mark.parametrize("it", [3.4e38, 2.4e38, 1e30, 1e-30, 1.4e-45])
@pytest.mark.parametrize("classes", [50, 5000, 140001])
def test_extreme_temperatures(classes, it):
    """Towards the largest class alone (ties share), and towards a uniform distribution: the largest finite fp32 numbers and the smallest one."""
    gen = torch.Generator().manual_seed(4)
    w = torch.randint(-3, 4, (5, classes), generator=gen).float()
    w[1] = torch.randn(classes, generator=gen)
    w[2, 1::2] = -math.inf
    w[3] = 2.0
    tokens = torch.tensor([0, int(w[1].argmax()), 0, 3, 1])
    dlp, dent = torch.ones(5), torch.zeros(5)
    it = float(torch.tensor(it))
    want = ref.logprob_forward(w.double(), it, None, tokens, 5)
    grad = ref.logprob_backward(w.double(), 1.0 if it > 1e38 else it, None, tokens, dlp.double(), dent.double())
    got = _run(w, classes, "f32", tokens, None, it, dlp, dent, 5)
    _same(got["logprob"], want["logprob"].float(), ABS, 1.0, "logprob")
    _same(got["entropy"], want["entropy"], ABS, 1.0, "entropy")
    assert torch.equal(got["top_index"].to(torch.int64), want["top_index"])
    _same(got["top_logprob"], want["top_logprob"].float(), ABS, 1.0, "top_logprob")
    assert not torch.isnan(got["dlogits"]).any()
    if 1e-20 < it < 1e38:
        _same(got["dlogits"], grad, ABS, float(grad.abs().max()), "dlogits")


@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_every_element_of_the_gradient_by_its_own_size(shape, dtype, masked):
    """dlogit = it (g [token] - p (g + h (log p + H))), an element at a time.  Exponents of up to some 30 are rounded two or three times (2^-24 of
    themselves each) and the sum by 1e-6, so p is good to 1e-5 of itself, and log p + H to 1e-5 of its terms; the token's g adds its own rounding of
    2^-22, and bf16 the last one of 2^-8."""
    rows, classes, pad = shape
    it = 0.8 if masked else 1.0
    wide, tokens, mask, it, dlp, dent = _case(rows, classes, pad, dtype, masked, sum(shape) + 1, it)
    got = _run(wide, classes, dtype, tokens, mask, it, dlp, dent, 0)["dlogits"].double()
    v = wide[:, :classes].double()
    if masked:
        v = v.masked_fill(~mask, -math.inf)
    empty = (v == -math.inf).all(1)
    z = torch.where(empty[:, None], torch.zeros(()).double(), v) * it
    logp = torch.log_softmax(z, 1)
    p = torch.exp(logp)
    logp = torch.where(p > 0, logp, torch.zeros(()).double())
    H = -(p * logp).sum(1, keepdim=True)
    given = (tokens >= 0) & (tokens < classes)
    g, h = torch.where(given, dlp, torch.zeros(())).double()[:, None], dent.double()[:, None]
    want = -p * (g + h * (logp + H))
    bound = 1e-5 * p * (g.abs() + h.abs() * (logp.abs() + H + 1))
    at = torch.zeros(rows, classes, dtype=torch.bool)
    at[given, tokens[given]] = True
    want = want + at * g
    bound = bound + at * g.abs() * 2.0 ** -22
    dead = empty[:, None] | (~mask if masked else torch.zeros(rows, classes, dtype=torch.bool))
    want, bound = torch.where(dead, torch.zeros(()).double(), want * it), torch.where(dead, torch.zeros(()).double(), bound * it)
    if dtype == "bf16":
        bound = bound + 2.0 ** -8 * want.abs()
    over = (got - want).abs() - bound
    assert float(over.max()) <= 1e-37, (float(over.max()), int(over.argmax()), float((over > 1e-37).double().mean()))
