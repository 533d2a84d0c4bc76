"""A gated pair of FCs and its gradients against the definition in 64 bits, element by element."""
import pytest
import torch

import more_operators_ref as ref
from paper_2304_07741_amd import binding as B
from paper_2304_07741_amd import harness

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
# rows, features, width: single ones, sizes that no tile, vector or wave divides, the borders of the path for few rows (16, 32), one tile and
# one more than it, sums of one step and of one more, sums cut into parts (many rows and few weights), tiles of 256
SHAPES = [(1, 1, 1), (1, 17, 3), (3, 5, 7), (4, 2048, 40), (16, 64, 33), (17, 136, 64), (32, 1001, 50), (33, 40, 24), (64, 64, 256), (128, 64, 64), (129, 72, 65),
          (130, 1000, 300), (257, 65, 129), (300, 128, 1), (1500, 8, 16), (9001, 64, 64), (5000, 100, 24)]
LARGE = [(3100, 72, 2000), (2900, 328, 1900), (700, 700, 6000), (1001, 1993, 8101)]


def _case(rows, features, width, dtype, seed, std=1.0):
    gen = torch.Generator().manual_seed(seed)
    dt = TYPES[dtype]
    make = lambda *s, k=1.0: (torch.randn(*s, generator=gen) * k).to(dt).cuda()  # noqa: E731
    return make(rows, features), make(width, features, k=std / features ** 0.5), make(width, features, k=std / features ** 0.5), make(rows, width)


def _run(rows, features, width, dtype, kind, tensors, flags=0):
    x, wg, wu, dy = tensors
    r = harness.GatedRunner(rows, features, width, dtype, kind, flags=flags)
    for t in [*r.out.values(), *r.grads.values()]:
        t.fill_(float("nan"))
    r.ws.fill_(0xFF)
    out = {k: v.clone() for k, v in r.forward(x, wg, wu).items()}
    if not flags:
        out |= {k: v.clone() for k, v in r.backward(x, wg, wu, dy).items()}
    torch.cuda.synchronize()
    r.close()
    return out


def _compare(got, val, bound, f32, what):
    for name, v in val.items():
        g = got[name].double()
        assert g.shape == v.shape and bool(torch.isfinite(g).all()), (what, name)
        over = (g - v).abs() - bound[name] - 1e-37
        assert float(over.max()) <= 0, (what, name, float((g - v).abs().max()), int((over > 0).sum()))
        # and over all elements: two roundings to the type, uniform within half a step each (rms half / 3^(1/2), both together 0.82 half at most), or
        # a sum in fp32.  A mean over n independent squares, of variance 4/5 of its own square each, is past 1.5 times its expectation (1 / 0.82^2)
        # by chance with 0.5 (n / 0.8)^(1/2) standard deviations: 17 of them for n = 1000, 2.6 for the 21 gradients of 3 rows of 7
        if f32 or got["y"].numel() >= 1000:
            rel = float((g - v).norm() / v.norm().clamp_min(1e-30))
            assert rel <= (2e-5 if f32 else 2.0 ** -8), (what, name, rel)


@pytest.mark.parametrize("kind", [B.CANVAS_GATED_SIGMOID, B.CANVAS_GATED_SILU, B.CANVAS_GATED_GELU], ids=["sigmoid", "silu", "gelu"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_against_the_definition(shape, dtype, kind):
    t = _case(*shape, dtype, 7 + sum(shape), std=2.0)
    val, bound = ref.gated(kind, *(v.double() for v in t), f32=dtype == "f32")
    _compare(_run(*shape, dtype, kind, t), val, bound, dtype == "f32", (shape, dtype, kind))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", LARGE, ids=str)
def test_large_tiles(shape, dtype):
    t = _case(*shape, dtype, 3)
    val, bound = ref.gated(B.CANVAS_GATED_SILU, *(v.double() for v in t), f32=dtype == "f32")
    _compare(_run(*shape, dtype, B.CANVAS_GATED_SILU, t), val, bound, dtype == "f32", (shape, dtype))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 1, 1), (5, 333, 70), (32, 64, 16), (40, 33, 70), (300, 512, 200)], ids=str)
def test_inference_plans_give_the_same(shape, dtype):
    t = _case(*shape, dtype, 11)
    full, infer = _run(*shape, dtype, B.CANVAS_GATED_GELU, t), _run(*shape, dtype, B.CANVAS_GATED_GELU, t, flags=B.CANVAS_OPT_INFERENCE)
    assert torch.equal(full["y"], infer["y"])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", [0, 1, 2])
def test_gates_far_from_zero(dtype, kind):
    """Gates from -200 to 200: the tails of the activations and of their slopes."""
    rows, features, width = 40, 8, 64
    dt = TYPES[dtype]
    x = torch.zeros(rows, features, device="cuda")
    x[:, 0] = torch.linspace(-200, 200, rows, device="cuda")
    x[:, 1] = 1
    wg = torch.zeros(width, features, device="cuda")
    wg[:, 0] = torch.linspace(0, 1, width, device="cuda")
    wu = torch.zeros(width, features, device="cuda")
    wu[:, 1] = torch.linspace(-3, 3, width, device="cuda")
    dy = torch.ones(rows, width, device="cuda")
    t = [v.to(dt) for v in (x, wg, wu, dy)]
    val, bound = ref.gated(kind, *(v.double() for v in t), f32=dtype == "f32")
    _compare(_run(rows, features, width, dtype, kind, t), val, bound, dtype == "f32", (dtype, kind))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [3, 50])
def test_what_is_not_finite_stays_in_its_rows(dtype, rows):
    """A NaN in a row of x makes that row of y and dx NaN and no other; one in a row of a weight its column of y."""
    features, width = 70, 90
    x, wg, wu, dy = _case(rows, features, width, dtype, 5)
    x[1, 3], wu[2, 5] = float("nan"), float("nan")
    got = _run(rows, features, width, dtype, 1, (x, wg, wu, dy))
    bad = torch.zeros(rows, width, dtype=torch.bool, device="cuda")
    bad[1], bad[:, 2] = True, True
    assert torch.equal(torch.isnan(got["y"]), bad)
    x[1, 3] = 0
    clean = _run(rows, features, width, dtype, 1, (x, wg, wu, dy))
    assert torch.equal(got["y"][~bad], clean["y"][~bad])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gradients_against_differences(dtype):
    """sum(y dy) from the kernels themselves, fp32: central differences along random directions."""
    if dtype == "bf16":
        pytest.skip("differences of values of 8 bits say nothing")
    shape = (70, 40, 56)
    x, wg, wu, dy = _case(*shape, dtype, 9)
    r = harness.GatedRunner(*shape, dtype, B.CANVAS_GATED_SILU)
    r.forward(x, wg, wu)
    g = {k: v.clone() for k, v in r.backward(x, wg, wu, dy).items()}
    gen = torch.Generator().manual_seed(1)
    for name, at in (("dx", 0), ("dw_gate", 1), ("dw_up", 2)):
        args = [x, wg, wu]
        v = torch.randn(args[at].shape, generator=gen).cuda()
        loss = []
        for s in (1, -1):
            moved = list(args)
            moved[at] = args[at] + s * 2.0 ** -8 * v
            loss.append(float((r.forward(*moved)["y"].double() * dy.double()).sum()))
        want, got = (loss[0] - loss[1]) / 2.0 ** -7, float((g[name].double() * v.double()).sum())
        # the third derivative's part: about 2^-16 of the sum's size; y's rounding: 2^-24 sqrt(70 56) |y dy| / 2^-8
        assert abs(want - got) <= 1e-3 * float(g[name].double().norm() * v.double().norm()) , (name, want, got)
    r.close()
