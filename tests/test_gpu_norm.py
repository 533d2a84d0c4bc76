"""The norms between two blocks against their definition in 64 bits."""
import math

import pytest
import torch

import operators_ref as ref
from helpers import TOL, assert_close
from paper_2304_07741_amd import binding as B
from paper_2304_07741_amd import harness

pytestmark = pytest.mark.gpu

BOTH = B.CANVAS_NORM_POST | B.CANVAS_NORM_PRE
# parts, gate
PLANS = [(BOTH, B.CANVAS_GATE_SILU), (BOTH, B.CANVAS_GATE_NONE), (B.CANVAS_NORM_PRE, B.CANVAS_GATE_NONE), (B.CANVAS_NORM_POST, B.CANVAS_GATE_SIGMOID)]
# one pixel and one channel; rows of tokens, short, odd and longer than a workgroup; planes from two pixels on: odd, of whole
# vectors, longer than a tile; few and many channels
SHAPES = [(1, 1, 1, 1), (3, 1, 2, 5), (1, 7, 1, 1), (5, 64, 1, 1), (37, 1000, 1, 1), (3, 4099, 1, 1), (2, 16384, 1, 1), (700, 48, 1, 1),
          (2, 33, 1, 2), (3, 8, 3, 1), (70, 24, 2, 2), (5, 64, 7, 7), (2, 257, 9, 13), (3, 96, 16, 16), (1, 16, 1, 4099), (2, 520, 14, 14), (1, 2100, 5, 8),
          (9, 40, 28, 28), (1, 5000, 3, 3)]
EPS = 1e-3


def _case(shape, dtype, parts, gate, seed, scale_x=1.0):
    n, c, h, w = shape
    gen = torch.Generator().manual_seed(seed)
    dt = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    maps = {k: (torch.randn(n, c, h, w, generator=gen) * s).to(dt) for k, s in (("x", scale_x), ("z", 0.7), ("g", 2.0), ("dy", 1.0), ("du", 1.0))}
    weights = {"w_post": torch.randn(c, generator=gen), "scale": torch.randn(c, generator=gen) * 0.5, "w_pre": torch.randn(c, generator=gen)}
    post, pre = bool(parts & B.CANVAS_NORM_POST), bool(parts & B.CANVAS_NORM_PRE)
    if not post:
        maps.pop("z"), weights.pop("w_post"), weights.pop("scale")
    if not gate:
        maps.pop("g")
    if not pre:
        weights.pop("w_pre"), maps.pop("du")
    return maps, weights


def _reference(shape, maps, weights, gate, with_dy):
    n, c, h, w = shape
    m = {k: v.double().reshape(n, c, h * w) for k, v in maps.items()}
    wt = {k: v.double() for k, v in weights.items()}
    y, u = ref.norm_forward(m["x"], m.get("z"), m.get("g"), wt.get("w_post"), wt.get("scale"), wt.get("w_pre"), gate, EPS)
    out = {"x_out": y, "u": u}
    out |= ref.norm_backward(y, m.get("z"), m.get("g"), wt.get("w_post"), wt.get("scale"), wt.get("w_pre"), gate, EPS, m["dy"] if with_dy else None, m.get("du"))
    return {k: v.numpy() for k, v in out.items() if v is not None}


def _run(shape, dtype, parts, gate, maps, weights, with_dy=True, device="cuda:0"):
    r = harness.NormRunner(shape, dtype, parts, gate=gate, eps=EPS)
    d = {k: v.to(device) for k, v in {**maps, **weights}.items()}
    for t in [*r.out.values(), *r.grads.values()]:
        t.fill_(float("nan"))
    r.ws.fill_(0xFF)
    block = (d.get("z"), d.get("g"), d.get("w_post"), d.get("scale"), d.get("w_pre"))
    out = r.forward(d["x"], *block)
    got = {**out, **r.backward(out.get("x_out", d["x"]), *block, dx_out=d["dy"] if with_dy else None, du=d.get("du"))}
    torch.cuda.synchronize()
    res = {k: v.double().cpu().numpy() for k, v in got.items()}
    r.close()
    return res


@pytest.mark.parametrize("parts,gate", PLANS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_forward_and_backward(shape, dtype, parts, gate):
    maps, weights = _case(shape, dtype, parts, gate, seed=sum(shape))
    want = _reference(shape, maps, weights, gate, True)
    got = _run(shape, dtype, parts, gate, maps, weights)
    n, c, h, w = shape
    for k, g in got.items():
        # the weights' gradients are fp32 sums of the operands as they were loaded; bf16 plans read x' rounded, which each of
        # the terms carries once: 2^-9 of a term, so the bound of the maps holds for their sum
        floor = 1e-2 if k in ("dz", "dw_post", "dscale", "dgate", "dx", "dw_pre") and c == 1 else 1e-30
        assert_close(g.reshape(want[k].shape), want[k], TOL[dtype], f"{shape} {dtype} {k}", floor=floor)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_no_gradient_on_the_stream_is_a_gradient_of_zeros(dtype):
    shape = (3, 48, 5, 7)
    maps, weights = _case(shape, dtype, BOTH, B.CANVAS_GATE_SILU, 11)
    want = _reference(shape, maps, weights, B.CANVAS_GATE_SILU, False)
    got = _run(shape, dtype, BOTH, B.CANVAS_GATE_SILU, maps, weights, with_dy=False)
    for k, g in got.items():
        assert_close(g.reshape(want[k].shape), want[k], TOL[dtype], k)


def test_pixels_of_zeros_and_of_large_values():
    """A pixel whose channels are all zero is divided by the root of eps; squares of 1e18 stay in range."""
    shape = (2, 64, 6, 6)
    for scale in (0.0, 1e-18, 1e15):
        maps, weights = _case(shape, "f32", BOTH, B.CANVAS_GATE_NONE, 5)
        maps["x"] = maps["x"] * scale
        maps["z"][0, :, 2, 3] = 0
        maps["x"][0, :, 2, 3] = 0
        want = _reference(shape, maps, weights, B.CANVAS_GATE_NONE, True)
        got = _run(shape, "f32", BOTH, B.CANVAS_GATE_NONE, maps, weights)
        for k in ("x_out", "u", "dx", "dz", "dw_pre"):
            assert_close(got[k].reshape(want[k].shape), want[k], TOL["f32"], f"{scale} {k}")


def test_a_pixel_with_nan_keeps_it_to_itself():
    shape = (2, 40, 7, 7)
    maps, weights = _case(shape, "bf16", BOTH, B.CANVAS_GATE_SIGMOID, 9)
    clean = _run(shape, "bf16", BOTH, B.CANVAS_GATE_SIGMOID, maps, weights)
    maps["z"][1, 3, 4, 5] = float("nan")
    got = _run(shape, "bf16", BOTH, B.CANVAS_GATE_SIGMOID, maps, weights)
    for k in ("x_out", "u", "dx", "dz", "dgate"):
        t = torch.from_numpy(got[k]).clone()
        assert torch.isnan(t[1, :, 4, 5]).any(), k
        t[1, :, 4, 5] = torch.from_numpy(clean[k])[1, :, 4, 5]
        assert torch.equal(t, torch.from_numpy(clean[k])), k


@pytest.mark.parametrize("shape", [(64, 64, 20, 20), (300, 512, 1, 1)])
def test_two_runs_and_two_streams_give_the_same_bits(shape):
    maps, weights = _case(shape, "bf16", BOTH, B.CANVAS_GATE_SILU, 2)
    first = _run(shape, "bf16", BOTH, B.CANVAS_GATE_SILU, maps, weights)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        again = _run(shape, "bf16", BOTH, B.CANVAS_GATE_SILU, maps, weights)
    for k in first:
        assert (first[k] == again[k]).all(), k


def test_inference_plan():
    shape = (4, 96, 7, 7)
    maps, weights = _case(shape, "bf16", BOTH, B.CANVAS_GATE_SILU, 4)
    want = _reference(shape, maps, weights, B.CANVAS_GATE_SILU, True)
    r = harness.NormRunner(shape, "bf16", BOTH, gate=B.CANVAS_GATE_SILU, eps=EPS, flags=B.CANVAS_OPT_INFERENCE)
    assert r.info.workspace_bytes == 0 and r.info.n_launches_bwd == 0
    d = {k: v.cuda() for k, v in {**maps, **weights}.items()}
    out = r.forward(d["x"], d["z"], d["g"], d["w_post"], d["scale"], d["w_pre"])
    for k, g in out.items():
        assert_close(g.double().cpu().numpy().reshape(want[k].shape), want[k], TOL["bf16"], k)
    with pytest.raises(B.CanvasError) as e:
        r.backward(out["x_out"], d["z"], d["g"], d["w_post"], d["scale"], d["w_pre"], dx_out=d["dy"], du=d["du"])
    assert e.value.status == -6
    r.close()


def test_gradient_against_differences_of_the_kernel():
    """(L(x + h d) - L(x - h d)) / 2h of the forward kernel.  Truncation ~ h^2 = 1e-4 of the value, the fp32 rounding of the
    outputs 1e-7 sqrt(n) / h ~ 1e-3 of a loss gradient of norm sqrt(n): 5e-3 bounds both."""
    shape, h = (2, 32, 4, 4), 1e-2
    maps, weights = _case(shape, "f32", BOTH, B.CANVAS_GATE_SILU, 21)
    got = _run(shape, "f32", BOTH, B.CANVAS_GATE_SILU, maps, weights)
    gen = torch.Generator().manual_seed(1)

    def loss(m, w):
        r = harness.NormRunner(shape, "f32", BOTH, gate=B.CANVAS_GATE_SILU, eps=EPS)
        d = {k: v.cuda() for k, v in {**m, **w}.items()}
        out = {k: v.double().cpu() for k, v in r.forward(d["x"], d["z"], d["g"], d["w_post"], d["scale"], d["w_pre"]).items()}
        r.close()
        return float((out["x_out"] * m["dy"].double()).sum() + (out["u"] * m["du"].double()).sum())

    for name, grad in (("x", "dx"), ("z", "dz"), ("g", "dgate"), ("w_post", "dw_post"), ("scale", "dscale"), ("w_pre", "dw_pre")):
        src = maps if name in maps else weights
        g = torch.from_numpy(got[grad])
        d = torch.randn(src[name].shape, generator=gen) * 0.1 + (g / g.norm()).float()
        d /= d.norm()
        up = {k: (v + h * d if k == name else v) for k, v in src.items()}
        down = {k: (v - h * d if k == name else v) for k, v in src.items()}
        pair = [loss(m, weights) if src is maps else loss(maps, m) for m in (up, down)]
        want, have = (pair[0] - pair[1]) / (2 * h), float((g * d.double()).sum())
        assert abs(want - have) <= 5e-3 * abs(have) + 5e-3, (name, want, have)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 1025, 3, 3), (2, 1500, 7, 7), (40, 2047, 3, 5), (70, 1030, 2, 13), (1, 2049, 7, 7), (33, 256, 7, 7)],
                         ids=lambda s: "x".join(map(str, s)))
def test_one_piece_of_a_plane_at_a_time(shape, dtype):
    """Many channels or few pixels: a workgroup holds all channels of one piece, or reads them again; with more pieces than workgroups."""
    for parts, gate in PLANS[:1] + PLANS[2:3]:
        maps, weights = _case(shape, dtype, parts, gate, seed=sum(shape))
        want = _reference(shape, maps, weights, gate, True)
        for k, g in _run(shape, dtype, parts, gate, maps, weights).items():
            assert_close(g.reshape(want[k].shape), want[k], TOL[dtype], f"{shape} {dtype} {k}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(64, 64, 16, 16), (64, 72, 19, 21), (64, 128, 19, 21), (64, 200, 16, 17), (48, 300, 21, 20)],
                         ids=lambda s: "x".join(map(str, s)))
def test_maps_that_fill_the_chip(shape, dtype):
    """Eight and four pieces of a plane side by side, forward and backward cut alike and differently, several tiles per workgroup."""
    for parts, gate in PLANS[:1] + PLANS[3:]:
        maps, weights = _case(shape, dtype, parts, gate, seed=sum(shape))
        want = _reference(shape, maps, weights, gate, True)
        for k, g in _run(shape, dtype, parts, gate, maps, weights).items():
            assert_close(g.reshape(want[k].shape), want[k], TOL[dtype], f"{shape} {dtype} {k}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(1100, 512, 1, 1), (1030, 2500, 1, 1), (520, 5120, 1, 1), (300, 8200, 1, 1)], ids=lambda s: "x".join(map(str, s)))
def test_rows_that_fill_the_chip(shape, dtype):
    """More rows than workgroups, by 64 to 1024 threads each."""
    maps, weights = _case(shape, dtype, BOTH, B.CANVAS_GATE_SILU, seed=sum(shape))
    want = _reference(shape, maps, weights, B.CANVAS_GATE_SILU, True)
    for k, g in _run(shape, dtype, BOTH, B.CANVAS_GATE_SILU, maps, weights).items():
        assert_close(g.reshape(want[k].shape), want[k], TOL[dtype], f"{shape} {dtype} {k}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(300, 24, 1, 3), (700, 24, 2, 3), (2000, 17, 2, 3), (1, 8, 56, 56), (5, 8, 56, 56), (9, 8, 56, 56), (2, 72, 56, 56),
                                   (5, 72, 56, 56), (1, 160, 56, 56), (1, 300, 56, 56), (1, 600, 56, 56), (260, 2049, 3, 3), (520, 2049, 3, 3), (1030, 2049, 3, 3)],
                         ids=lambda s: "x".join(map(str, s)))
def test_every_way_of_cutting_maps(shape, dtype):
    maps, weights = _case(shape, dtype, BOTH, B.CANVAS_GATE_SIGMOID, seed=sum(shape))
    want = _reference(shape, maps, weights, B.CANVAS_GATE_SIGMOID, True)
    for k, g in _run(shape, dtype, BOTH, B.CANVAS_GATE_SIGMOID, maps, weights).items():
        assert_close(g.reshape(want[k].shape), want[k], TOL[dtype], f"{shape} {dtype} {k}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_more_and_more_channels_in_one_process(dtype):
    """Sums of 8200 channels take 64 KB of LDS and more, of 16384 twice as much: the later plan is not held to what the first one took."""
    for shape in [(1, 8200, 3, 3), (2, 16384, 3, 3), (3, 12000, 1, 2), (2, 16384, 2, 1)]:
        maps, weights = _case(shape, dtype, BOTH, B.CANVAS_GATE_SILU, seed=sum(shape))
        want = _reference(shape, maps, weights, B.CANVAS_GATE_SILU, True)
        for k, g in _run(shape, dtype, BOTH, B.CANVAS_GATE_SILU, maps, weights).items():
            assert_close(g.reshape(want[k].shape), want[k], TOL[dtype], f"{shape} {dtype} {k}")


@pytest.mark.parametrize("scale,eps", [(1e15, 1e-3), (1e18, 1e-3), (1e-13, 1e-30), (0.0, 1e-30)])
@pytest.mark.parametrize("shape", [(2, 64, 6, 6), (3, 200, 1, 1), (1, 2100, 3, 3), (2, 16, 1, 2), (2, 5000, 1, 1)], ids=lambda s: "x".join(map(str, s)))
def test_gradients_of_maps_far_from_one(shape, scale, eps):
    """The third power of 1 / |x'| leaves the range of fp32 long before the gradient does, which falls and rises as the first one."""
    maps, weights = _case(shape, "f32", BOTH, B.CANVAS_GATE_SILU, 6)
    maps["x"], maps["z"] = maps["x"] * scale, maps["z"] * scale
    weights["scale"] = weights["scale"] * max(scale, 1e-20)          # (x' is of the size of x)
    n, c, h, w = shape
    m = {k: v.double().reshape(n, c, h * w) for k, v in maps.items()}
    wt = {k: v.double() for k, v in weights.items()}
    y, _ = ref.norm_forward(m["x"], m["z"], m["g"], wt["w_post"], wt["scale"], wt["w_pre"], B.CANVAS_GATE_SILU, eps)
    want = ref.norm_backward(y, m["z"], m["g"], wt["w_post"], wt["scale"], wt["w_pre"], B.CANVAS_GATE_SILU, eps, None, m["du"])
    r = harness.NormRunner(shape, "f32", BOTH, gate=B.CANVAS_GATE_SILU, eps=eps)
    d = {k: v.cuda() for k, v in {**maps, **weights}.items()}
    block = (d["z"], d["g"], d["w_post"], d["scale"], d["w_pre"])
    out = r.forward(d["x"], *block)
    got = r.backward(out["x_out"], *block, du=d["du"])
    for k in ("dx", "dz", "dgate", "dw_pre"):
        assert_close(got[k].double().cpu().numpy().reshape(want[k].shape), want[k].numpy(), TOL["f32"], f"{scale} {k}")
    r.close()


@pytest.mark.parametrize("gate", [B.CANVAS_GATE_SIGMOID, B.CANVAS_GATE_SILU])
@pytest.mark.parametrize("shape", [(1, 64, 9, 10), (90, 64, 1, 1), (2, 30, 32, 3), (3, 2100, 1, 3)], ids=lambda s: "x".join(map(str, s)))
def test_gates_to_a_few_units(shape, gate):
    """x = 0, z = 1 and weights of one leave x' = act(gate), and a gradient of ones leaves dgate = act'(gate).  Exponential and reciprocal are good to a unit each
    (2^-23), 1 + e^-g, the root and the products to half of one: 6e-7 in all, held to 8e-7 from gates of -80 on.  (The slope by its
    terms' size: it is a difference.)"""
    n = shape[0] * shape[1] * shape[2] * shape[3]
    g = torch.linspace(-80, 20, n).reshape(shape)
    one, w = torch.ones(shape), torch.ones(shape[1])
    r = harness.NormRunner(shape, "f32", B.CANVAS_NORM_POST, gate=gate, eps=1e-12)
    out = r.forward(torch.zeros(shape).cuda(), one.cuda(), g.cuda(), w.cuda(), w.cuda())
    x_out = out["x_out"].double().cpu()
    dgate = r.backward(out["x_out"], one.cuda(), g.cuda(), w.cuda(), w.cuda(), dx_out=one.cuda())["dgate"].double().cpu()
    a, slope = ref.act(gate, g.double())
    assert float(((x_out - a).abs() / a.abs().clamp(min=1e-38)).max()) <= 8e-7
    s = torch.sigmoid(g.double())
    size = s if gate == B.CANVAS_GATE_SIGMOID else s * (1 + g.double().abs())
    assert float(((dgate - slope).abs() / size).max()) <= 8e-7
    r.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 16, 4, 8), (2, 16, 1, 1)], ids=lambda s: "x".join(map(str, s)))
def test_infinite_gates_and_nan(shape, dtype):
    """A sigmoid gate of -inf shuts, of +inf opens and passes no gradient on; NaN stays NaN, where it is."""
    dt = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    g = torch.zeros(shape)
    g[0, 0], g[0, 1], g[0, 2], g[0, 3], g[0, 4] = -math.inf, math.inf, math.nan, -1e38, 1e38
    one, w = torch.ones(shape, dtype=dt, device="cuda"), torch.ones(shape[1], device="cuda")
    r = harness.NormRunner(shape, dtype, B.CANVAS_NORM_POST, gate=B.CANVAS_GATE_SIGMOID, eps=1e-12)
    out = r.forward(torch.zeros(shape, dtype=dt, device="cuda"), one, g.to(dt).cuda(), w, w)
    x = out["x_out"].float().cpu()
    d = r.backward(out["x_out"], one, g.to(dt).cuda(), w, w, dx_out=one)["dgate"].float().cpu()
    assert (x[0, [0, 3]] == 0).all() and ((x[0, [1, 4]] - 1).abs() < 1e-6).all() and torch.isnan(x[0, 2]).all()
    assert (d[0, [0, 1, 3, 4]] == 0).all() and torch.isnan(d[0, 2]).all()
    assert ((x[0, 5:] - 0.5).abs() < 1e-6).all() and ((d[0, 5:] - 0.25).abs() < 1e-6).all()
    r.close()


@pytest.mark.parametrize("parts,gate", PLANS)
@pytest.mark.parametrize("shape", [(5, 64, 1, 1), (37, 1000, 1, 1), (3, 4099, 1, 1), (2, 16384, 1, 1), (700, 48, 1, 1), (2, 33, 1, 2), (70, 24, 2, 2), (5, 64, 7, 7), (2, 257, 9, 13),
                                   (3, 96, 16, 16), (2, 520, 14, 14), (1, 2100, 5, 8), (9, 40, 28, 28), (64, 64, 16, 16)], ids=lambda s: "x".join(map(str, s)))
def test_weight_gradients_of_bf16_plans_are_fp32(shape, parts, gate):
    """They are fp32 sums of what the bf16 maps hold, x' among it before its rounding: held to the bound of fp32 plans."""
    maps, weights = _case(shape, "bf16", parts, gate, seed=sum(shape) + 1)
    want = _reference(shape, maps, weights, gate, True)
    got = _run(shape, "bf16", parts, gate, maps, weights)
    for k in ("dw_post", "dscale", "dw_pre"):
        if k in got:
            assert_close(got[k].reshape(want[k].shape), want[k], TOL["f32"], f"{shape} {k}")
