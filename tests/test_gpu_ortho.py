"""Orthogonalised updates against the definition in 64 bits."""
import math

import pytest
import torch

import operators_ref as ref
from paper_2304_07741_amd import binding as B
from paper_2304_07741_amd import harness

pytestmark = pytest.mark.gpu

# one element; one row, one column; grouped FCs; odd sides; sides around 16, 32, 64 and 128; tall ones; many small matrices
SHAPES = [(1, 1, 1), (3, 1, 7), (2, 9, 1), (8, 8, 72), (1, 16, 16), (5, 17, 33), (1, 72, 8), (2, 64, 576), (1, 63, 65), (1, 64, 640), (3, 65, 130), (1, 130, 300),
          (1, 129, 129), (1, 300, 130), (70, 40, 10), (1, 256, 2304), (1, 33, 5000), (2, 200, 1031), (1, 640, 200), (1, 520, 776), (1, 1100, 1300)]

# Each operand of a product carries 22 bits and sums are fp32: 2^-22 of the largest singular value.  Five steps raise what a
# weak direction holds by at most 3.4445^5 = 485 while the strongest stays near one, so an error grows to 485 * 2^-22 = 1.2e-4.
TOL_F32 = 1.2e-4
TOL_BF16 = TOL_F32 + 2.0 ** -8


def _inputs(shape, seed, kind="noise"):
    gen = torch.Generator().manual_seed(seed)
    g, r, k = shape
    grad = torch.randn(g, r, k, generator=gen)
    if kind == "low":
        rank = max(1, min(r, k) // 8)
        grad = torch.randn(g, r, rank, generator=gen) @ torch.randn(g, rank, k, generator=gen) + 0.05 * grad
    return grad, torch.randn(g, r, k, generator=gen), torch.randn(g, r, k, generator=gen)


def _err(got, want):
    got, want = got.double().cpu(), want.double()
    assert torch.isfinite(got).all()
    return max(float((got - want).norm() / want.norm().clamp(min=1e-30)), float((got - want).abs().max() / want.abs().max().clamp(min=1e-30)))


def _step(shape, dtype, grad, momentum=None, master=None, mu=0.9, lr=0.02, decay=0.1, steps=5, flags=0):
    r = harness.OrthoRunner(shape, dtype, steps=steps, flags=flags)
    r.ws.fill_(0xFF)
    r.out["update"].fill_(float("nan"))
    d = [None if t is None else t.cuda() for t in (grad, momentum, master)]
    out = {k: v.cpu() for k, v in r.step(*d, mu=mu, lr=lr, decay=decay).items()}
    r.close()
    return out


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["noise", "low"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_step(shape, kind, dtype):
    grad, momentum, master = _inputs(shape, sum(shape), kind)
    momentum = momentum * 0.1
    tol = TOL_F32 if dtype == "f32" else TOL_BF16
    nesterov = sum(shape) % 2 == 0
    want = ref.ortho_step(grad.double(), momentum.double(), 0.9, nesterov, 5, master.double(), 0.02, 0.1)
    got = _step(shape, dtype, grad, momentum, master, flags=B.CANVAS_ORTHO_NESTEROV if nesterov else 0)
    assert _err(got["update"], want["update"]) <= tol
    assert _err(got["momentum"], want["momentum"]) <= 1e-6
    assert _err(got["master"], want["master"]) <= 0.02 * TOL_F32 + 1e-6
    assert torch.equal(got["weights"], got["master"].to(got["weights"].dtype))


@pytest.mark.parametrize("steps", [0, 1, 2, 8])
@pytest.mark.parametrize("shape", [(2, 24, 40), (1, 150, 70), (1, 260, 300)])
def test_number_of_steps(shape, steps):
    grad, _, _ = _inputs(shape, 3)
    want = ref.ortho_step(grad.double(), None, 0, False, steps)
    got = _step(shape, "f32", grad, steps=steps)
    assert set(got) == {"update"} and _err(got["update"], want["update"]) <= TOL_F32 * max(1, steps / 5)


@pytest.mark.parametrize("scale", [1e-30, 1e-7, 1e25])
@pytest.mark.parametrize("shape", [(2, 24, 40), (1, 200, 300)])
def test_gradients_of_any_size(shape, scale):
    grad, _, _ = _inputs(shape, 4)
    grad = grad * scale
    want = ref.ortho_step(grad.double(), None, 0, False, 5)
    got = _step(shape, "f32", grad)["update"].double()
    # (1e-30: the division by |v| + 1e-7 leaves 1e-22 and less, which the fp16 pairs do not hold: zeros to that accuracy)
    assert torch.isfinite(got).all() and float((got - want["update"]).norm()) <= TOL_F32 * max(1.0, float(want["update"].norm()))


@pytest.mark.parametrize("shape", [(4, 24, 40), (4, 130, 200)])
def test_zeros_and_nan_stay_in_their_matrix(shape):
    grad, _, _ = _inputs(shape, 5)
    clean = _step(shape, "f32", grad)["update"]
    grad[1] = 0
    grad[2, 3, 5] = math.nan
    got = _step(shape, "f32", grad)["update"]
    assert (got[1] == 0).all() and torch.isnan(got[2]).any()
    assert torch.equal(got[0], clean[0]) and torch.equal(got[3], clean[3])
    grad[2, 3, 5] = math.inf
    got = _step(shape, "f32", grad)["update"]
    assert torch.isnan(got[2]).any() and torch.equal(got[0], clean[0]) and torch.equal(got[3], clean[3])


@pytest.mark.parametrize("shape", [(3, 40, 56), (1, 256, 300)])
def test_in_place_and_on_another_stream(shape):
    """momentum_out = momentum and master_out = master give the bits of separate tensors; so does a second stream."""
    grad, momentum, master = _inputs(shape, 6)
    a = _step(shape, "bf16", grad, momentum, master)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        r = harness.OrthoRunner(shape, "bf16")
        g, m, w = grad.cuda(), momentum.cuda(), master.cuda()
        u, p = r.out["update"], torch.empty(shape, dtype=torch.bfloat16, device="cuda")
        B.canvas_ortho_step(r.handle, g, m, m, 0.9, w, w, 0.02, 0.1, p, u, r.ws)
        side.synchronize()
    for k, t in (("update", u), ("momentum", m), ("master", w), ("weights", p)):
        assert torch.equal(a[k], t.cpu()), k
    # without an update tensor
    m, w = momentum.cuda(), master.cuda()
    B.canvas_ortho_step(r.handle, g, m, m, 0.9, w, w, 0.02, 0.1, None, None, r.ws)
    torch.cuda.synchronize()
    assert torch.equal(a["master"], w.cpu())
    r.close()


@pytest.mark.parametrize("shape", [(4, 1100, 3300), (4, 3300, 1100), (4, 1024, 1500), (300, 100, 90)], ids=lambda s: "x".join(map(str, s)))
def test_many_tiles(shape):
    """Tiles of every size, with and without sums in parts; the definition in 64 bits is computed on the GPU."""
    grad, _, _ = _inputs(shape, 8, "low")
    d = grad.double().cuda()
    want = torch.stack([ref.newton_schulz(m, 5) for m in d]).cpu()
    assert _err(_step(shape, "f32", grad)["update"], want) <= TOL_F32


@pytest.mark.parametrize("steps", [1, 2, 3, 4, 5])
@pytest.mark.parametrize("shape", [(1, 100, 450), (2, 500, 90), (3, 65, 1031)], ids=lambda s: "x".join(map(str, s)))
def test_two_steps_at_a_time(shape, steps):
    """One side several times the other: pairs of steps are joined, and an odd one is left at the end."""
    for kind in ("noise", "low"):
        grad, _, _ = _inputs(shape, 9 + steps, kind)
        want = ref.ortho_step(grad.double(), None, 0, False, steps)
        assert _err(_step(shape, "f32", grad, steps=steps)["update"], want["update"]) <= TOL_F32


@pytest.mark.parametrize("shape", [(1, 1700, 6200), (14, 1250, 1300), (2, 1600, 3300), (6, 700, 720)], ids=lambda s: "x".join(map(str, s)))
def test_large_tiles(shape):
    """Symmetric products by tiles of 256 and 128, whole and in parts; the definition in 64 bits is computed on the GPU."""
    grad, _, _ = _inputs(shape, 9, "low")
    d = grad.double().cuda()
    want = torch.stack([ref.newton_schulz(m, 5) for m in d]).cpu()
    assert _err(_step(shape, "f32", grad)["update"], want) <= TOL_F32


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_larger_and_larger_small_matrices_in_one_process(dtype):
    """63 x 65 takes 73 KB of LDS, 64 x 256 118: the later plan is not held to what the first one took."""
    for shape in [(2, 63, 65), (1, 64, 256), (2, 48, 480), (1, 480, 48)]:
        grad, _, _ = _inputs(shape, 10)
        want = ref.ortho_step(grad.double(), None, 0, False, 5)
        assert _err(_step(shape, dtype, grad)["update"], want["update"]) <= (TOL_F32 if dtype == "f32" else TOL_BF16)


@pytest.mark.parametrize("scale", [1e-38, 1e-30, 1e-20, 1e-14, 1e-12, 1e-11, 1e-10, 1e-9, 1.0, 1e30])
@pytest.mark.parametrize("shape", [(2, 24, 40), (2, 200, 300), (2, 100, 450), (2, 300, 130), (1, 520, 776)], ids=lambda s: "x".join(map(str, s)))
def test_gradients_of_any_size_to_the_same_relative_accuracy(shape, scale):
    """|v| + 1e-7 leaves X small where |v| is, down to 1e-31; every matrix of a call has a size of its own."""
    grad, _, _ = _inputs(shape, 12)
    grad = grad * scale
    if shape[0] > 1:
        grad[1] *= 1e-3 if scale > 1e-30 else 1e3
    for steps in (5, 2):
        want = ref.ortho_step(grad.double(), None, 0, False, steps)["update"]
        got = _step(shape, "f32", grad, steps=steps)["update"]
        for g, w in zip(got, want):
            assert float(w.norm()) > 0 and _err(g, w) <= TOL_F32


@pytest.mark.parametrize("scale", [1e-25, 1e-12])
@pytest.mark.parametrize("shape", [(1, 1700, 6200), (1, 2600, 1300), (14, 1250, 1300)], ids=lambda s: "x".join(map(str, s)))
def test_small_gradients_in_large_tiles(shape, scale):
    """The definition in 64 bits is computed on the GPU."""
    grad, _, _ = _inputs(shape, 13)
    grad = grad * scale
    d = grad.double().cuda()
    want = torch.stack([ref.newton_schulz(m, 5) for m in d]).cpu()
    assert _err(_step(shape, "f32", grad)["update"], want) <= TOL_F32


@pytest.mark.parametrize("steps", [0, 1, 5])
@pytest.mark.parametrize("shape", [(3, 24, 40), (3, 130, 200), (3, 100, 450)], ids=lambda s: "x".join(map(str, s)))
def test_an_infinity_makes_its_whole_matrix_nan(shape, steps):
    grad, _, _ = _inputs(shape, 14)
    clean = _step(shape, "f32", grad, steps=steps)["update"]
    for v in (math.inf, -math.inf, math.nan):
        grad[1, 3, 5] = v
        got = _step(shape, "f32", grad, steps=steps)["update"]
        assert torch.isnan(got[1]).all()
        assert torch.equal(got[0], clean[0]) and torch.equal(got[2], clean[2])


@pytest.mark.parametrize("shape", [(2, 24, 40), (1, 64, 576), (1, 130, 300), (1, 256, 2304), (1, 300, 130), (2, 200, 1031), (1, 640, 200), (1, 520, 776), (2, 90, 3000)],
                         ids=lambda s: "x".join(map(str, s)))
def test_operands_hold_all_their_bits(shape):
    """Matrices without weak directions: their singular values lie within a factor of ten, so a step keeps relative errors about as they are, and five
    steps of three products whose operands are good to 2^-22 leave 15 times that, 4e-6, and sums in fp32 half as much again.  (A model in 64 bits with five bits of the lower halves lost is
    9e-6 to 2e-5 off.)"""
    grad, _, _ = _inputs(shape, 15)
    want = ref.ortho_step(grad.double(), None, 0, False, 5)["update"]
    assert _err(_step(shape, "f32", grad)["update"], want) <= 6e-6


@pytest.mark.parametrize("span", [1.0, 1e-3, 1e-6])
@pytest.mark.parametrize("shape", [(1, 24, 40), (1, 48, 80), (1, 64, 200), (1, 16, 300), (1, 200, 300), (1, 300, 200), (1, 128, 1024), (1, 520, 776)], ids=lambda s: "x".join(map(str, s)))
def test_as_exact_as_products_in_fp32(shape, span):
    """Singular values from one down to `span`, evenly on their logarithm: no more than half as much again as the formula's error with products in fp32."""
    gen = torch.Generator().manual_seed(16)
    side = min(shape[1:])
    u, _ = torch.linalg.qr(torch.randn(shape[1], side, generator=gen, dtype=torch.float64))
    v, _ = torch.linalg.qr(torch.randn(shape[2], side, generator=gen, dtype=torch.float64))
    grad = ((u * torch.logspace(0, math.log10(span), side, dtype=torch.float64)) @ v.T).float()[None]
    want = ref.newton_schulz(grad[0].double(), 5)
    x = (grad[0] / (grad[0].norm() + 1e-7)).cuda()
    x = x.T.contiguous() if shape[1] > shape[2] else x
    a, b, c = ref.COEFFICIENTS
    for _ in range(5):
        q = x @ x.T.contiguous()
        x = a * x + (b * q + c * (q @ q)) @ x
    x = x.T if shape[1] > shape[2] else x
    off = lambda t: float((t.double().cpu() - want).norm() / want.norm())  # noqa: E731
    assert off(_step(shape, "f32", grad)["update"][0]) <= 1.5 * off(x) + 1e-7
