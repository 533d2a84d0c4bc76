"""The norm over many tensors and their scaling against 64 bits."""
import math

import pytest
import torch

import more_operators_ref as ref
from paper_2304_07741_amd import binding as B
from paper_2304_07741_amd import harness

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
# counts of the tensors: one element, no vector whole, one chunk of 8192 and its neighbours, empty ones between others, more than one launch takes, more
# chunks than workgroups
COUNTS = [[1], [7, 1, 9], [8192], [8191, 8193, 0, 16384], [0, 5, 0], [3] * 97, [40000, 3, 12345, 64] * 60, [20_000_003], [9_000_000, 1, 3_000_001]]


def _grads(counts, kinds, seed, std=1e-2):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return [(torch.randn(n, generator=gen, device="cuda") * std * (1 + i % 5)).to(TYPES[k]) for i, (n, k) in enumerate(zip(counts, kinds))]


def _check(got, grads, most):
    norm, scale, want = ref.clip(grads, most)
    # the norm: one rounding of a sum in 64 bits; the scale: that of its own; an element: scale and product in fp32, and its type
    assert abs(float(got["norm"]) - norm) <= 2.0 ** -24 * norm * 1.01
    assert abs(float(got["scale"]) - scale) <= 2.0 ** -24 * scale * 1.01
    for g, w in zip(got["grads"], want):
        half = 2.0 ** -8 if g.dtype is torch.bfloat16 else 2.0 ** -24
        assert g.numel() == 0 or float(((g.double() - w).abs() - (half + 2.0 ** -23) * 1.01 * w.abs()).max()) <= 1e-40


@pytest.mark.parametrize("out", ["same", "f32", "bf16"])
@pytest.mark.parametrize("kind", ["f32", "bf16", "mixed"])
@pytest.mark.parametrize("counts", COUNTS, ids=lambda c: f"{len(c)}x{max(c)}")
def test_against_the_definition(counts, kind, out):
    kinds = [("f32", "bf16")[i % 2] for i in range(len(counts))] if kind == "mixed" else [kind] * len(counts)
    grads = _grads(counts, kinds, len(counts))
    r = harness.ClipRunner([(n,) for n in counts], kinds, None if out == "same" else [out] * len(counts))
    for most in (ref.clip(grads, 1.0)[0] * 0.3, 1e6, math.inf):
        r.ws.fill_(0xFF)
        _check(r.step(grads, most), grads, most)
    r.close()


@pytest.mark.parametrize("kind", ["f32", "bf16", "mixed"])
def test_in_place_and_the_norm_alone(kind):
    counts = [1000, 8193, 3, 100_000]
    kinds = [("f32", "bf16")[i % 2] for i in range(4)] if kind == "mixed" else [kind] * 4
    grads = _grads(counts, kinds, 3)
    before = [g.clone() for g in grads]
    r = harness.ClipRunner([(n,) for n in counts], kinds)
    norm = torch.zeros((), device="cuda")
    B.canvas_clip_step(r.handle, grads, None, 1.0, norm, None, r.ws)
    assert abs(float(norm) - ref.clip(before, 1.0)[0]) <= 1e-6 * float(norm)
    assert all(torch.equal(a, b) for a, b in zip(grads, before))
    apart = [g.clone() for g in r.step(grads, 0.25)["grads"]]
    _check(r.step(grads, 0.25, in_place=True), before, 0.25)
    assert all(torch.equal(a, b) for a, b in zip(grads, apart))
    again = [g.clone() for g in grads]
    r.step(grads, 1e9, in_place=True)
    assert all(torch.equal(a, b) for a, b in zip(grads, again))
    r.close()


@pytest.mark.parametrize("offset", [1, 2, 3, 5])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_tensors_that_begin_anywhere(kind, offset):
    base = _grads([30_000 + offset], [kind], offset)[0]
    grads = [base[offset:]]
    r = harness.ClipRunner([(30_000,)], [kind])
    _check(r.step(grads, 0.5), grads, 0.5)
    want = r.step(grads, 0.5)["grads"][0].clone()
    kept = base[:offset].clone()
    r.step(grads, 0.5, in_place=True)
    assert torch.equal(base[offset:], want) and torch.equal(base[:offset], kept)
    r.close()


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_largest_and_smallest_values(kind):
    """Squares far outside fp32, and a scale below its smallest normal number."""
    dt = TYPES[kind]
    for value in (3e38, 1e-38, 1e-30, 2.0 ** 100):
        g = [torch.full((5000,), value, device="cuda").to(dt), torch.full((77,), -value, device="cuda").to(dt)]
        r = harness.ClipRunner([(5000,), (77,)], [kind] * 2, ["f32"] * 2)
        for most in (1e-2, 1e-35):
            norm, scale, want = ref.clip(g, most)
            got = r.step(g, most)
            assert float(got["norm"]) == pytest.approx(norm if norm < 3.4028235e38 else math.inf, rel=2e-7)    # (as fp32 holds it)
            for a, b in zip(got["grads"], want):
                assert float(((a.double() - b).abs() - 2.0 ** -22 * b.abs()).max()) <= 1e-44
        r.close()


def test_what_is_not_finite():
    g = _grads([3000, 50], ["f32", "bf16"], 1)
    r = harness.ClipRunner([(3000,), (50,)], ["f32", "bf16"])
    g[1][7] = math.nan
    got = r.step(g, 1.0)
    assert math.isnan(float(got["norm"])) and math.isnan(float(got["scale"])) and all(bool(torch.isnan(t).all()) for t in got["grads"])
    g[1][7] = math.inf
    got = r.step(g, 1.0)
    assert float(got["norm"]) == math.inf and float(got["scale"]) == 0
    assert not got["grads"][0].any() and int(torch.isnan(got["grads"][1]).sum()) == 1 and float(got["grads"][1].nan_to_num().abs().max()) == 0
    g = [torch.zeros(3000, device="cuda"), torch.zeros(50, device="cuda").bfloat16()]
    got = r.step(g, 1.0)
    assert float(got["norm"]) == 0 and float(got["scale"]) == 1 and not got["grads"][0].any()
    r.close()
