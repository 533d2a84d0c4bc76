"""Host-only checks of gated pairs, heads without logits and the clipping of gradients: exported names, queries and refusals.  No GPU is needed: a
call is refused before anything is launched."""
import ctypes
import os
import re

import pytest
import torch

from paper_2304_07741_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def P(k):
    """Aligned addresses far apart that no refused call looks at."""
    return (k + 1) << 40


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        import __graft_entry__ as g

        g.build()
    return B.load()


def _status(f, *a, **k):
    with pytest.raises(B.CanvasError) as e:
        f(*a, **k)
    assert str(e.value)
    return e.value.status


@pytest.mark.parametrize("header,names", [("canvas_gated.h", B.GATED_EXPORTS), ("canvas_head.h", B.HEAD_EXPORTS), ("canvas_clip.h", B.CLIP_EXPORTS)])
def test_every_declared_symbol_is_exported(lib, header, names):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", header)).read(), flags=re.S)
    assert set(re.findall(r"\b(canvas_[a-z_]+)\s*\(", text)) == set(names)
    for name in names:
        assert getattr(lib, name) is not None


# ---------------------------------------------------------------- gated pairs

def test_gated_compile_and_query(lib):
    h = B.canvas_gated_compile(100, 64, 256, B.CANVAS_BF16, B.CANVAS_GATED_GELU)
    info = B.canvas_gated_query(h)
    assert info.n_launches_fwd >= 1 and info.n_launches_bwd >= 2 and info.workspace_bytes >= 4 * 100 * 256
    assert info.flops_fwd == 4.0 * 100 * 64 * 256 and info.flops_bwd == 2 * info.flops_fwd
    assert info.min_bytes_fwd == 2.0 * (100 * 64 + 2 * 64 * 256 + 100 * 256)
    B.canvas_gated_destroy(h)
    h = B.canvas_gated_compile(100, 64, 256, B.CANVAS_BF16, flags=B.CANVAS_OPT_INFERENCE)
    assert B.canvas_gated_query(h).n_launches_bwd == 0
    assert lib.canvas_gated_backward(h, *[P(k) for k in range(8)], 1 << 30, None) == -6
    B.canvas_gated_destroy(h)
    B.canvas_gated_destroy(None)


@pytest.mark.parametrize("kw,status", [
    ({"rows": 0}, -4), ({"features": 0}, -4), ({"width": -1}, -4), ({"rows": 1 << 31}, -6), ({"features": B.CANVAS_GATED_MAX_SIDE + 1}, -6),
    ({"width": B.CANVAS_GATED_MAX_SIDE + 1}, -6), ({"dtype": 2}, -4), ({"act": 3}, -4), ({"act": -1}, -4), ({"flags": 1}, -4), ({"flags": 4}, -4),
    ({"rows": (1 << 31) - 1, "width": 1 << 18}, -6)])
def test_gated_compile_refuses(lib, kw, status):
    a = {"rows": 3, "features": 4, "width": 5, "dtype": 0, "act": 1, "flags": 0, **kw}
    assert _status(B.canvas_gated_compile, a["rows"], a["features"], a["width"], a["dtype"], a["act"], a["flags"]) == status


def test_gated_calls_refuse(lib):
    h = B.canvas_gated_compile(100, 64, 256, B.CANVAS_F32)
    ws = B.canvas_gated_query(h).workspace_bytes
    for call, n in ((lib.canvas_gated_forward, 5), (lib.canvas_gated_backward, 8)):
        good = [P(k) for k in range(n)]
        for k in range(n):
            for bad in (None, P(k) + 8):
                a = list(good)
                a[k] = bad
                assert call(h, *a, ws, None) == -4 and lib.canvas_last_error()
        assert call(h, *good, ws - 1, None) == -5
        assert call(None, *good, ws, None) == -4
    # what is written shares bytes with something: forward's y, backward's three gradients, the workspace
    for call, n, written in ((lib.canvas_gated_forward, 5, (3, 4)), (lib.canvas_gated_backward, 8, (4, 5, 6, 7))):
        for k in written:
            for other in range(n):
                if other != k:
                    a = [P(i) for i in range(n)]
                    a[k] = a[other] + 16
                    assert call(h, *a, ws, None) == -4, (k, other)
    B.canvas_gated_destroy(h)
    assert lib.canvas_gated_query(None, ctypes.byref(B.CanvasGatedInfo())) == -4


# ---------------------------------------------------------------- heads

def test_head_compile_and_query(lib):
    h = B.canvas_head_compile(1000, 64, 5000, B.CANVAS_BF16)
    info = B.canvas_head_query(h)
    assert info.n_launches_fwd >= 2 and info.n_launches_bwd >= 3 and info.pieces >= 1
    assert info.flops_fwd == 2.0 * 1000 * 64 * 5000 and info.flops_bwd == 3 * info.flops_fwd
    B.canvas_head_destroy(h)
    # the logits of 2^16 rows x 2^18 classes would take 32 GB: the workspace holds a piece of them
    h = B.canvas_head_compile(1 << 16, 1024, 1 << 18, B.CANVAS_BF16)
    info = B.canvas_head_query(h)
    assert info.pieces > 50 and info.workspace_bytes < (1 << 16) * (1 << 18) * 2 // 8
    B.canvas_head_destroy(h)
    h = B.canvas_head_compile(10, 64, 5000, B.CANVAS_F32, flags=B.CANVAS_OPT_INFERENCE)
    assert B.canvas_head_query(h).n_launches_bwd == 0
    assert lib.canvas_head_backward(h, P(0), P(1), 1.0, None, P(2), P(3), P(4), P(5), P(6), P(7), 1 << 30, None) == -6
    B.canvas_head_destroy(h)
    B.canvas_head_destroy(None)


@pytest.mark.parametrize("kw,status", [
    ({"rows": 0}, -4), ({"features": 0}, -4), ({"classes": 0}, -4), ({"rows": 1 << 31}, -6), ({"features": B.CANVAS_HEAD_MAX_FEATURES + 1}, -6),
    ({"classes": B.CANVAS_HEAD_MAX_CLASSES + 1}, -6), ({"dtype": 2}, -4), ({"flags": 1}, -4), ({"rows": (1 << 31) - 1, "classes": 1 << 20}, -6)])
def test_head_compile_refuses(lib, kw, status):
    a = {"rows": 3, "features": 4, "classes": 5, "dtype": 0, "flags": 0, **kw}
    assert _status(B.canvas_head_compile, a["rows"], a["features"], a["classes"], a["dtype"], a["flags"]) == status


def test_head_calls_refuse(lib):
    h = B.canvas_head_compile(100, 64, 500, B.CANVAS_F32)
    ws = B.canvas_head_query(h).workspace_bytes

    def forward(x=P(0), w=P(1), it=1.0, mask=P(2), tokens=P(3), logprob=P(4), entropy=P(5), space=P(6), n=ws):
        return lib.canvas_head_forward(h, x, w, it, mask, tokens, logprob, entropy, space, n, None)

    def backward(x=P(0), w=P(1), it=1.0, mask=P(2), tokens=P(3), dlp=P(4), dent=P(5), dx=P(6), dw=P(7), space=P(8), n=ws):
        return lib.canvas_head_backward(h, x, w, it, mask, tokens, dlp, dent, dx, dw, space, n, None)

    for it in (0.0, -1.0, float("nan"), float("inf")):
        assert forward(it=it) == -4 and backward(it=it) == -4
    for name in ("x", "w", "tokens", "logprob", "space"):
        assert forward(**{name: None}) == -4
    for name in ("x", "w", "mask", "tokens", "logprob", "entropy", "space"):
        assert forward(**{name: P(20) + 8}) == -4
    for name in ("x", "w", "tokens", "dx", "dw", "space"):
        assert backward(**{name: None}) == -4
    for name in ("x", "w", "mask", "tokens", "dlp", "dent", "dx", "dw", "space"):
        assert backward(**{name: P(20) + 8}) == -4
    assert forward(n=ws - 1) == -5 and backward(n=ws - 1) == -5
    for name, others in (("logprob", "x w mask tokens entropy space"), ("entropy", "x w mask tokens logprob space"), ("space", "x w mask tokens")):
        for other in others.split():
            assert forward(**{name: P(30), other: P(30) + 16}) == -4, (name, other)
    for name in ("dx", "dw", "space"):
        for other in "x w mask tokens dlp dent dx dw space".split():
            if other != name:
                assert backward(**{name: P(30), other: P(30) + 16}) == -4, (name, other)
    B.canvas_head_destroy(h)
    assert lib.canvas_head_query(None, ctypes.byref(B.CanvasHeadInfo())) == -4


# ---------------------------------------------------------------- clipping

def _clip(counts, types, outs=None):
    return B.canvas_clip_compile(counts, types, outs)


def test_clip_compile_and_query(lib):
    h = _clip([100, 0, 7], [0, 1, 1], [0, 1, 0])
    info = B.canvas_clip_query(h)
    assert info.n_launches >= 1 and info.workspace_bytes >= 8 and info.min_bytes == 100 * 8 + 7 * 6
    B.canvas_clip_destroy(h)
    h = _clip([5] * 1000, [0] * 1000)
    assert B.canvas_clip_query(h).n_launches <= 2 * 11 + 1
    B.canvas_clip_destroy(h)
    B.canvas_clip_destroy(None)


@pytest.mark.parametrize("counts,types,outs,status", [
    ([], [], None, -4), ([-1], [0], None, -4), ([1], [2], None, -4), ([1], [0], [3], -4), ([(1 << 40) + 1], [0], None, -6), ([1 << 40] * 16, [0] * 16, None, -6),
    ([1] * 65537, [0] * 65537, None, -6)], ids=range(7))
def test_clip_compile_refuses(lib, counts, types, outs, status):
    assert _status(_clip, counts, types, outs) == status
    assert lib.canvas_clip_compile(1, None, (ctypes.c_int * 1)(0), None, ctypes.byref(ctypes.c_void_p())) == -4
    with pytest.raises(ValueError):
        _clip([1, 2], [0])


def test_clip_calls_refuse(lib):
    h = _clip([100, 0, 50], [0, 0, 1], [0, 0, 0])
    ws = B.canvas_clip_query(h).workspace_bytes
    array = lambda v: (ctypes.c_void_p * len(v))(*v)  # noqa: E731

    def step(grads=(P(0), None, P(1)), outs=(P(2), None, P(3)), most=1.0, norm=P(4), scale=P(5), space=P(6), n=ws):
        return lib.canvas_clip_step(h, None if grads is None else array(grads), None if outs is None else array(outs), most, norm, scale, space, n, None)

    assert step(grads=None) == -4 and step(norm=None) == -4 and step(space=None) == -4 and step(n=ws - 1) == -5
    for most in (0.0, -1.0, float("nan")):
        assert step(most=most) == -4
    assert step(grads=(None, None, P(1))) == -4 and step(outs=(P(2), None, None)) == -4
    assert step(grads=(P(0) + 2, None, P(1))) == -4 and step(grads=(P(0), None, P(1) + 1)) == -4 and step(outs=(P(2), None, P(3) + 2)) == -4
    assert step(norm=P(4) + 2) == -4 and step(scale=P(5) + 1) == -4
    assert step(outs=(P(0), None, P(1))) == -4                   # the second has another type than its out
    assert step(outs=(P(0) + 4, None, P(3))) == -4               # not the same place, and not apart from it
    assert step(outs=(P(1), None, P(3))) == -4                   # over another gradient
    assert step(grads=(P(0), None, P(0)), outs=(P(0), None, P(3))) == -4
    assert step(outs=(P(2), None, P(2) + 396)) == -4             # outs over each other
    assert step(norm=P(0)) == -4 and step(scale=P(4)) == -4 and step(scale=P(2) + 396) == -4 and step(space=P(1)) == -4 and step(space=P(4) - 16) == -4
    B.canvas_clip_destroy(h)
    # the same tensor twice: scaled twice in its place, so refused
    h = _clip([100, 100], [0, 0])
    assert lib.canvas_clip_step(h, array((P(0), P(0))), array((P(0), P(0))), 1.0, P(4), None, P(6), 1 << 20, None) == -4
    B.canvas_clip_destroy(h)
    assert lib.canvas_clip_query(None, ctypes.byref(B.CanvasClipInfo())) == -4


def test_clip_step_wants_as_many_tensors_as_its_plan_has(lib):
    h = B.canvas_clip_compile([8, 8], [B.CANVAS_F32] * 2)
    t = torch.zeros(8)
    for grads, outs in (([t], None), ([t] * 3, [t] * 3), ([t] * 2, [t])):
        with pytest.raises(ValueError, match="2 tensors are needed"):
            B.canvas_clip_step(h, grads, outs, 1.0, t[:1], None, t)
    B.canvas_clip_destroy(h)
