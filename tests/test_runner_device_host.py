"""Runners call the library with their own device as the current one, whichever was current before: an address of one GPU in a launch on another is a fault.  No GPU
is needed: tensors are the host's, and the library's calls are recorded."""
import pytest
import torch

from paper_2304_07741_amd import binding as B
from paper_2304_07741_amd import harness

CALLS = ["canvas_norm_forward", "canvas_norm_backward", "canvas_logprob_forward", "canvas_logprob_backward", "canvas_ortho_step", "canvas_gated_forward", "canvas_gated_backward",
         "canvas_head_forward", "canvas_head_backward", "canvas_clip_step"]


def _use(r):
    z = torch.zeros
    if isinstance(r, harness.NormRunner):
        r.backward(r.forward(z(2, 4, 3, 3), w_pre=z(4)) and r.passed, w_pre=z(4), du=z(2, 4, 3, 3))
    elif isinstance(r, harness.LogprobRunner):
        t = z(3, dtype=torch.int64)
        r.forward(z(3, 5), t)
        r.backward(z(3, 5), t, z(3))
    elif isinstance(r, harness.OrthoRunner):
        r.step(z(1, 4, 6))
    elif isinstance(r, harness.GatedRunner):
        x, w = z(3, 4), z(5, 4)
        r.forward(x, w, w)
        r.backward(x, w, w, z(3, 5))
    elif isinstance(r, harness.HeadRunner):
        x, w, t = z(3, 4), z(5, 4), z(3, dtype=torch.int64)
        r.forward(x, w, t)
        r.backward(x, w, t, z(3))
    else:
        r.step([z(7)], 1.0)


MAKE = {"norm": lambda: harness.NormRunner((2, 4, 3, 3), "f32", B.CANVAS_NORM_PRE, device="cpu"), "logprob": lambda: harness.LogprobRunner(3, 5, "f32", device="cpu"),
        "ortho": lambda: harness.OrthoRunner((1, 4, 6), "f32", device="cpu"), "gated": lambda: harness.GatedRunner(3, 4, 5, "f32", device="cpu"),
        "head": lambda: harness.HeadRunner(3, 4, 5, "f32", device="cpu"), "clip": lambda: harness.ClipRunner([(7,)], ["f32"], device="cpu")}


@pytest.mark.parametrize("name", MAKE)
def test_calls_are_made_on_the_runners_device(name, monkeypatch):
    current, calls = [0], []

    class Device:
        def __init__(self, device):
            self.device = device

        def __enter__(self):
            self.before, current[0] = current[0], self.device

        def __exit__(self, *error):
            current[0] = self.before

    monkeypatch.setattr(torch.cuda, "is_available", lambda: True)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(harness, "_current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "device", Device)
    for f in CALLS:
        monkeypatch.setattr(B, f, lambda *a, f=f: calls.append((f, current[0])))
    r = MAKE[name]()
    r.device = torch.device("cpu")       # of no number, so not the current one
    _use(r)
    assert len(calls) == (1 if name in ("ortho", "clip") else 2) and all(d == r.device for _, d in calls), calls
    assert current == [0]
    r.close()
