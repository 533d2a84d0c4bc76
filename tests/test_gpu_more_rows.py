"""Heads of more rows than a launch has workgroups, whatever a workgroup takes of them."""
import pytest
import torch

from paper_2304_07741_amd import binding as B
from paper_2304_07741_amd import harness

pytestmark = pytest.mark.gpu


def _taken(values, at):
    """values[at], a part of `at` at a time: torch's indexing gives zeros for some rows of results of more than 2^30 elements."""
    out = torch.empty(at.shape[0], *values.shape[1:], dtype=values.dtype, device=values.device)
    for part in range(0, at.shape[0], 1 << 24):
        out[part:part + (1 << 24)] = values[at[part:part + (1 << 24)]]
    return out


def test_rows_beyond_two_to_the_28():
    """The launch that joins a row's sums has 16 rows a workgroup and 2^24 - 1 workgroups along x: with more, every row has the bits of a plan of 112 rows, gradients too."""
    rows, features, classes = (1 << 28) + 5, 8, 5
    if torch.cuda.mem_get_info()[0] < 64 << 30:
        pytest.skip("64 GiB of the GPU's memory are needed")
    gen = torch.Generator(device="cuda")
    gen.manual_seed(6)
    x, w = torch.randn(14, features, generator=gen, device="cuda").bfloat16(), torch.randn(classes, features, generator=gen, device="cuda").bfloat16()
    tokens, d = torch.arange(14, device="cuda") % 6 - 1, torch.randn(14, generator=gen, device="cuda")
    at, many = torch.arange(112, device="cuda") % 14, torch.arange(rows, device="cuda") % 14
    small, large = harness.HeadRunner(112, features, classes, "bf16"), harness.HeadRunner(rows, features, classes, "bf16")
    large.ws.fill_(0xFF)
    for t in [*large.out.values(), *large.grads.values()]:
        t.fill_(float("nan"))
    for r, which in ((small, at), (large, many)):
        a = (_taken(x, which), w, _taken(tokens, which))
        r.forward(*a)
        r.backward(*a, *[_taken(d, which)] * 2)
    for name, got, want in [("logprob", large.out["logprob"], small.out["logprob"]), ("entropy", large.out["entropy"], small.out["entropy"]), ("dx", large.grads["dx"], small.grads["dx"])]:
        for part in range(0, rows, 1 << 24):
            assert torch.equal(got[part:part + (1 << 24)], want[:14][many[part:part + (1 << 24)]]), (name, part)
    small.close()
    large.close()
