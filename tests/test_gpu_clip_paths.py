"""Clipping on every way through its launches: one workgroup, workgroups that each add the sums up, a launch of its own for that, results past the last-level cache."""
import math

import pytest
import torch

import more_operators_ref as ref
from paper_2304_07741_amd import binding as B
from paper_2304_07741_amd import harness

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
# counts and launches of a call that writes: one launch; two, of one batch and of several; several batches with more sums than every workgroup adds by itself
WAYS = {"one": ([3000, 50], 1), "two": ([30000, 50, 16385], 2), "batches": ([400] * 100 + [20000], 4), "alone": ([16385] * 1100 + [3] * 2100, 2 * 34 + 1)}


def _runner(counts, kinds, outs=None):
    return harness.ClipRunner([(n,) for n in counts], kinds, outs)


def _same(got, want, half):
    return got.numel() == 0 or float(((got.double() - want).abs() - (half + 2.0 ** -23) * 1.01 * want.abs()).max()) <= 1e-40


def _check(got, grads, most):
    norm, scale, want = ref.clip(grads, most)
    assert abs(float(got["norm"]) - norm) <= 2.0 ** -24 * norm * 1.01
    assert abs(float(got["scale"]) - scale) <= 2.0 ** -24 * scale * 1.01
    for g, w in zip(got["grads"], want):
        assert _same(g, w, 2.0 ** -8 if g.dtype is torch.bfloat16 else 2.0 ** -24)


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("way", WAYS)
def test_every_way_against_the_definition(way, out):
    counts, launches = WAYS[way]
    kinds = [("f32", "bf16")[i % 2] for i in range(len(counts))]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    grads = [(torch.randn(n, generator=gen, device="cuda") * (1 + i % 5)).to(TYPES[k]) for i, (n, k) in enumerate(zip(counts, kinds))]
    r = _runner(counts, kinds, [out] * len(counts))
    assert r.info.n_launches == launches
    for most in (3.0, 1e9, math.inf):
        r.ws.fill_(0xFF)
        _check(r.step(grads, most), grads, most)
    r.close()


@pytest.mark.parametrize("count", [16383, 16384, 16385, 32769])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_borders_of_a_chunk(kind, count):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(count)
    grads = [torch.randn(n, generator=gen, device="cuda").to(TYPES[kind]) for n in (count, 0, 16384, count)]
    r = _runner([count, 0, 16384, count], [kind] * 4)
    _check(r.step(grads, 1.0), grads, 1.0)
    before = [g.clone() for g in grads]
    _check(r.step(grads, 2.0, in_place=True), before, 2.0)
    r.close()


@pytest.mark.parametrize("value", [3e38, 1e-38, 1e-30, 2.0 ** 100])
@pytest.mark.parametrize("way", WAYS)
def test_largest_and_smallest_values(way, value):
    """Squares far outside fp32, and a scale below its smallest normal number."""
    counts, _ = WAYS[way]
    kinds = [("f32", "bf16")[i % 2] for i in range(len(counts))]
    g = [torch.full((n,), value if i % 3 else -value, device="cuda").to(TYPES[k]) for i, (n, k) in enumerate(zip(counts, kinds))]
    r = _runner(counts, kinds, ["f32"] * len(counts))
    for most in (1e-2, 1e-35):
        norm, _, want = ref.clip(g, most)
        got = r.step(g, most)
        assert float(got["norm"]) == pytest.approx(norm if norm < 3.4028235e38 else math.inf, rel=2e-7)
        for a, b in zip(got["grads"], want):
            assert float(((a.double() - b).abs() - 2.0 ** -22 * b.abs()).max()) <= 1e-44
    r.close()


@pytest.mark.parametrize("way", WAYS)
def test_what_is_not_finite(way):
    counts, _ = WAYS[way]
    kinds = [("f32", "bf16")[i % 2] for i in range(len(counts))]
    g = [torch.ones(n, device="cuda").to(TYPES[k]) for n, k in zip(counts, kinds)]
    r = _runner(counts, kinds)
    g[1][1] = math.nan
    for most in (1.0, 1.75e308):
        got = r.step(g, most)
        assert math.isnan(float(got["norm"])) and math.isnan(float(got["scale"])) and all(bool(torch.isnan(t).all()) for t in got["grads"]), most
    g[1][1] = -math.inf
    for most in (1.0, 1.75e308):
        got = r.step(g, most)
        assert float(got["norm"]) == math.inf and float(got["scale"]) == 0, most
        assert not any(bool(t.any()) for k, t in enumerate(got["grads"]) if k != 1)
        assert int(torch.isnan(got["grads"][1]).sum()) == 1 and not bool(got["grads"][1].nan_to_num().any())
    for v in g:
        v.zero_()
    got = r.step(g, 1.0)
    assert float(got["norm"]) == 0 and float(got["scale"]) == 1 and not any(bool(t.any()) for t in got["grads"])
    r.close()


@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("way", WAYS)
def test_a_largest_norm_of_infinity_scales_nothing(way, value):
    """The norm tells what is not finite; every element stays what it is, in the type that it is asked for in."""
    counts, _ = WAYS[way]
    kinds = [("f32", "bf16")[i % 2] for i in range(len(counts))]
    g = [torch.full((n,), 1.5, device="cuda").to(TYPES[k]) for n, k in zip(counts, kinds)]
    g[1][2] = value
    r = _runner(counts, kinds, ["f32"] * len(counts))
    got = r.step(g, math.inf)
    assert torch.equal(got["norm"].cpu(), torch.tensor(abs(value))) or (math.isnan(value) and math.isnan(float(got["norm"])))
    assert float(got["scale"]) == 1
    assert all(torch.equal(a.view(torch.int32)[keep], b.float().view(torch.int32)[keep]) for a, b in zip(got["grads"], g) for keep in [~torch.isnan(b)])
    assert math.isnan(float(got["grads"][1][2])) == math.isnan(value)
    r.close()


@pytest.mark.parametrize("kind,out", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16"), ("f32", "bf16")])
def test_results_that_go_past_the_last_level_cache(kind, out):
    """More than 768 MiB read and written."""
    each = (4 if kind == "f32" else 2) + (4 if out == "f32" else 2)
    n = (800 << 20) // each
    counts = [n // 2 + 3, 5, 0, n // 2 - 16384]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(2)
    grads = [torch.randn(c, generator=gen, device="cuda").to(TYPES[kind]) for c in counts]
    r = _runner(counts, [kind] * 4, [out] * 4)
    assert r.info.min_bytes > 768 << 20
    _check(r.step(grads, 5.0), grads, 5.0)
    if kind == out:
        before = [g.clone() for g in grads]
        _check(r.step(grads, 5.0, in_place=True), before, 5.0)
    r.close()
