"""Host-only checks of the operators around a block: exported names, queries and refusals.  No GPU is needed: a call is refused
before anything is launched."""
import os
import re

import pytest

from paper_2304_07741_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BOTH = B.CANVAS_NORM_POST | B.CANVAS_NORM_PRE
P = 4096  # an aligned address that no refused call looks at


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        import __graft_entry__ as g

        g.build()
    return B.load()


@pytest.mark.parametrize("header,names", [("canvas_norm.h", B.NORM_EXPORTS), ("canvas_logprob.h", B.LOGPROB_EXPORTS), ("canvas_ortho.h", B.ORTHO_EXPORTS)])
def test_every_declared_symbol_is_exported(lib, header, names):
    text = open(os.path.join(ROOT, "include", header)).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    declared = set(re.findall(r"\b(canvas_[a-z_]+)\s*\(", text))
    assert declared == set(names)
    for name in names:
        assert getattr(lib, name) is not None


def _status(f, *a, **k):
    with pytest.raises(B.CanvasError) as e:
        f(*a, **k)
    assert str(e.value)
    return e.value.status


def test_norm_compile_and_query(lib):
    h = B.canvas_norm_compile((2, 64, 7, 7), B.CANVAS_BF16, BOTH, B.CANVAS_GATE_SILU)
    info = B.canvas_norm_query(h)
    e = 2.0 * 2 * 64 * 49
    assert info.n_launches_fwd >= 1 and info.n_launches_bwd >= 1 and info.workspace_bytes >= 8 * 64
    assert info.min_bytes_fwd == 5 * e and info.min_bytes_bwd == 8 * e
    B.canvas_norm_destroy(h)
    h = B.canvas_norm_compile((2, 64, 7, 7), B.CANVAS_F32, B.CANVAS_NORM_PRE, flags=B.CANVAS_OPT_INFERENCE)
    assert B.canvas_norm_query(h).workspace_bytes == 0
    B.canvas_norm_destroy(h)


@pytest.mark.parametrize("kw,status", [
    ({"shape": (0, 4, 1, 1)}, -4), ({"shape": (1, 4, 1, -1)}, -4), ({"shape": (1, B.CANVAS_NORM_MAX_CHANNELS + 1, 1, 1)}, -6),
    ({"shape": (1 << 20, 4, 1 << 20, 1)}, -6), ({"shape": (1, 4, 1 << 31, 1)}, -6), ({"dtype": 7}, -4), ({"parts": 0}, -4), ({"parts": 4}, -4), ({"gate": 3}, -4),
    ({"parts": B.CANVAS_NORM_PRE, "gate": 1}, -4), ({"eps": 0.0}, -4), ({"eps": -1.0}, -4), ({"eps": float("nan")}, -4), ({"eps": float("inf")}, -4),
    ({"flags": B.CANVAS_OPT_NO_FUSION}, -4)])
def test_norm_compile_refuses(lib, kw, status):
    a = {"shape": (1, 4, 2, 2), "dtype": B.CANVAS_F32, "parts": BOTH, "gate": 0, "eps": 1e-6, "flags": 0, **kw}
    assert _status(B.canvas_norm_compile, a["shape"], a["dtype"], a["parts"], a["gate"], a["eps"], a["flags"]) == status


def test_norm_calls_refuse(lib):
    h = B.canvas_norm_compile((2, 8, 3, 3), B.CANVAS_F32, BOTH, B.CANVAS_GATE_SIGMOID)
    ws = B.canvas_norm_query(h).workspace_bytes
    fwd = [P] * 9                                # x, z, gate, w_post, scale, w_pre, x_out, u, workspace
    for k in range(9):
        for bad in (None, P + 8):
            a = list(fwd)
            a[k] = bad
            assert lib.canvas_norm_forward(h, *a, ws, None) == -4 and lib.canvas_last_error()
    assert lib.canvas_norm_forward(h, *fwd, ws - 1, None) == -5
    assert lib.canvas_norm_forward(None, *fwd, ws, None) == -4
    # x, z, gate, w_post, scale, w_pre, dx_out, du, dx, dz, dgate, dw_post, dscale, dw_pre, workspace
    for k in range(15):
        for bad in ((None, P + 8) if k != 6 else (P + 8,)):
            a = [P] * 15
            a[k] = bad
            assert lib.canvas_norm_backward(h, *a, ws, None) == -4
    assert lib.canvas_norm_backward(h, *[P] * 15, ws - 1, None) == -5
    B.canvas_norm_destroy(h)
    h = B.canvas_norm_compile((2, 8, 3, 3), B.CANVAS_F32, B.CANVAS_NORM_POST)
    a = [P] * 15
    a[6] = None                                  # without PRE the gradient on the stream is the only one
    assert lib.canvas_norm_backward(h, *a, 1 << 20, None) == -4
    B.canvas_norm_destroy(h)
    h = B.canvas_norm_compile((2, 8, 3, 3), B.CANVAS_F32, BOTH, flags=B.CANVAS_OPT_INFERENCE)
    assert lib.canvas_norm_backward(h, *[P] * 15, 1 << 20, None) == -6
    B.canvas_norm_destroy(h)
    assert lib.canvas_norm_query(None, None) == -4
    B.canvas_norm_destroy(None)


def test_logprob_compile_and_query(lib):
    h = B.canvas_logprob_compile(5, 1000, B.CANVAS_BF16, 3)
    info = B.canvas_logprob_query(h)
    assert info.n_launches_fwd >= 1 and info.n_launches_bwd >= 1 and info.workspace_bytes >= 5 * 8
    assert info.min_bytes_fwd >= 10000 and info.min_bytes_bwd >= 20000
    B.canvas_logprob_destroy(h)


@pytest.mark.parametrize("a,status", [((0, 5, 0, 0, 0), -4), ((5, 0, 0, 0, 0), -4), ((1 << 31, 5, 0, 0, 0), -6), ((5, 1 << 31, 0, 0, 0), -6), ((5, 5, 9, 0, 0), -4),
                                      ((5, 5, 0, -1, 0), -4), ((5, 5, 0, B.CANVAS_LOGPROB_MAX_TOP + 1, 0), -4), ((5, 5, 0, 0, 1), -4)])
def test_logprob_compile_refuses(lib, a, status):
    assert _status(B.canvas_logprob_compile, *a) == status


def test_logprob_calls_refuse(lib):
    h = B.canvas_logprob_compile(5, 100, B.CANVAS_BF16, 3)
    ws = B.canvas_logprob_query(h).workspace_bytes

    def forward(logits=P, pitch=100, it=1.0, mask=None, mask_pitch=0, tokens=P, logprob=P, entropy=P, top=P, index=P, w=P, size=ws):
        return lib.canvas_logprob_forward(h, logits, pitch, it, mask, mask_pitch, tokens, logprob, entropy, top, index, w, size, None)

    for kw in ({"logits": None}, {"logits": P + 1}, {"pitch": 99}, {"pitch": -100}, {"pitch": 1 << 62}, {"it": 0.0}, {"it": -1.0}, {"it": float("nan")}, {"it": float("inf")},
               {"mask": P, "mask_pitch": 99}, {"mask": P, "mask_pitch": -1}, {"tokens": None}, {"tokens": P + 8}, {"logprob": None}, {"entropy": P + 4},
               {"top": None}, {"index": None}, {"w": None}, {"w": P + 8}):
        assert forward(**kw) == -4, kw
        assert lib.canvas_last_error()
    assert forward(size=ws - 1) == -5

    def backward(logits=P, pitch=100, it=1.0, mask=None, mask_pitch=0, tokens=P, dlp=P, dent=P, dl=2 * P, dpitch=100, w=P, size=ws):
        return lib.canvas_logprob_backward(h, logits, pitch, it, mask, mask_pitch, tokens, dlp, dent, dl, dpitch, w, size, None)

    for kw in ({"logits": None}, {"pitch": 99}, {"it": 0.0}, {"mask": P, "mask_pitch": 1}, {"tokens": None}, {"dlp": P + 4}, {"dent": P + 4}, {"dl": None}, {"dl": P + 1},
               {"dpitch": 99}, {"dl": P, "dpitch": 101}, {"w": None}):
        assert backward(**kw) == -4, kw
    assert backward(size=ws - 1) == -5
    B.canvas_logprob_destroy(h)
    h = B.canvas_logprob_compile(5, 100, B.CANVAS_BF16, 0, B.CANVAS_OPT_INFERENCE)
    assert lib.canvas_logprob_backward(h, P, 100, 1.0, None, 0, P, P, P, 2 * P, 100, P, 1 << 20, None) == -6
    B.canvas_logprob_destroy(h)
    assert lib.canvas_logprob_query(None, None) == -4
    B.canvas_logprob_destroy(None)


def test_ortho_compile_and_query(lib):
    h = B.canvas_ortho_compile((2, 8, 72), B.CANVAS_F32)
    info = B.canvas_ortho_query(h)
    assert info.flops == 2 * 5 * (8 * 9 * 72 + 8 * 9 * 8 + 2 * 64 * 72) and info.n_launches >= 1 and info.workspace_bytes >= 0
    B.canvas_ortho_destroy(h)


@pytest.mark.parametrize("a,status", [(((0, 4, 4), 0, 5, 0), -4), (((1, 4, -4), 0, 5, 0), -4), (((1, 4, 4), 3, 5, 0), -4), (((1, 4, 4), 0, -1, 0), -4),
                                      (((1, 4, 4), 0, B.CANVAS_ORTHO_MAX_STEPS + 1, 0), -4), (((1, 4, 4), 0, 5, 2), -4), (((1, 1 << 16, 1 << 16), 0, 5, 0), -6),
                                      (((1 << 30, 4, 4), 0, 5, 0), -6), (((1, B.CANVAS_ORTHO_MAX_SIDE + 1, B.CANVAS_ORTHO_MAX_SIDE + 1), 0, 5, 0), -6)])
def test_ortho_compile_refuses(lib, a, status):
    assert _status(B.canvas_ortho_compile, *a) == status


def test_ortho_calls_refuse(lib):
    h = B.canvas_ortho_compile((2, 8, 72), B.CANVAS_BF16)
    ws = B.canvas_ortho_query(h).workspace_bytes

    def step(grad=P, m=P, m_out=P, mu=0.9, w=P, w_out=P, lr=0.1, decay=0.0, weights=P, update=P, space=P, size=ws):
        return lib.canvas_ortho_step(h, grad, m, m_out, mu, w, w_out, lr, decay, weights, update, space, size, None)

    for kw in ({"grad": None}, {"grad": P + 4}, {"m": None}, {"m_out": None}, {"m": P + 4}, {"mu": 1.0}, {"mu": -0.1}, {"mu": float("nan")}, {"w": None}, {"w_out": None},
               {"lr": float("nan")}, {"decay": float("inf")}, {"weights": P + 2}, {"update": P + 2}, {"w": None, "w_out": None}, {"w": None, "w_out": None, "weights": None, "update": None},
               {"space": None}, {"space": P + 8}):
        assert step(**kw) == -4, kw
        assert lib.canvas_last_error()
    assert step(size=ws - 1) == -5
    assert lib.canvas_ortho_step(None, P, None, None, 0.0, None, None, 0.0, 0.0, None, P, P, ws, None) == -4
    B.canvas_ortho_destroy(h)
    assert lib.canvas_ortho_query(None, None) == -4
    B.canvas_ortho_destroy(None)


def test_stream_without_torchs_short_cut(monkeypatch):
    """The current stream's address comes from torch's public interface where the functions without checks are missing."""
    import torch

    monkeypatch.setattr(B, "_current_stream", None, raising=False)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: type("Stream", (), {"cuda_stream": 12345}))
    for name in ("_cuda_getCurrentRawStream", "_cuda_getDevice"):
        monkeypatch.delattr(torch._C, name, raising=False)
    assert B._stream() == 12345
    monkeypatch.setattr(B, "_current_stream", None, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 3, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 1000 + device, raising=False)
    assert B._stream() == 1003
