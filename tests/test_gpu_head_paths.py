"""Heads on ways that other tests pass by: masked classes in several pieces of a weight that is read as it is, logits that forward leaves of some pieces, backward
after a backward pass of other rows."""
import pytest
import torch

import more_operators_ref as ref
from paper_2304_07741_amd import harness
from test_gpu_head import _case, _check, _run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape", [(40000, 40, 4000), (9000, 64, 17001)], ids=str)
def test_masked_classes_in_several_pieces(shape):
    """bf16, features a multiple of 8: every piece's weight is copied without its masked classes, to one place."""
    plan = harness.HeadRunner(*shape, "bf16")
    assert plan.info.pieces > 1
    plan.close()
    case = _case(*shape, "bf16", 5, True)
    hidden = (~case[3]).nonzero()[:, 0]
    _check(case, "bf16", 1.0, shape)
    want = _run(*case, "bf16")
    case[1][hidden[0]], case[1][hidden[-1]] = float("nan"), float("inf")
    got = _run(*case, "bf16")
    assert all(torch.equal(got[k], want[k]) for k in want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_logits_of_the_first_pieces_are_left(dtype):
    """Many features, more logits than are left for backward: the first pieces are read, the others computed again."""
    shape = (20000, 1040, 14000) if dtype == "f32" else (24000, 2056, 12000)
    plan = harness.HeadRunner(*shape, dtype)
    assert plan.info.pieces > 1 and 4 * shape[0] * shape[2] > 1 << 30
    plan.close()
    _check(_case(*shape, dtype, 9, True), dtype, 0.8, shape)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(6, 100, 900), (200, 65, 1000), (200, 64, 1000), (5000, 40, 300)], ids=str)
def test_backward_after_one_of_other_rows(shape, dtype):
    """Rows without a gradient are zeros in what a backward pass leaves in the workspace: the next one, of all rows, gives what it gives by itself."""
    x, w, tokens, mask, a, b = _case(*shape, dtype, 4, True)
    want = _run(x, w, tokens, mask, a, b, dtype)
    r = harness.HeadRunner(*shape, dtype)
    r.forward(x, w, tokens, mask=mask)
    some = tokens.clone()
    some[::2] = -1
    first = {k: v.clone() for k, v in r.backward(x, w, some, a, None, mask=mask).items()}
    assert not first["dx"][::2].any() and first["dx"].any()
    for _ in range(2):
        got = r.backward(x, w, tokens, a, b, mask=mask)
        assert torch.equal(got["dx"], want["dx"]) and torch.equal(got["dweight"], want["dweight"])
        again = r.backward(x, w, some, a, None, mask=mask)
        assert torch.equal(again["dx"], first["dx"]) and torch.equal(again["dweight"], first["dweight"])
    r.close()


@pytest.mark.parametrize("value", [float("nan"), float("-inf")])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [9, 150])
def test_an_allowed_class_that_is_not_finite(rows, dtype, value):
    """One element of a weight: zero times it is NaN in that element of dx, of rows without a gradient too, and of no other element where the logits stay numbers."""
    x, w, tokens, _, a, _ = _case(rows, 40, 300, dtype, 4, False)
    x, tokens[0] = x.abs() + 0.5, 7                        # (logits of -inf, not of +inf)
    tokens[tokens == 5] = 6
    w[5, 3] = value
    got = _run(x, w, tokens, None, a, None, dtype)
    assert bool(torch.isnan(got["dx"][:, 3]).all())
    if value == value and dtype == "bf16":
        keep = torch.arange(40, device="cuda") != 3
        assert bool(torch.isfinite(got["logprob"]).all()) and bool(torch.isfinite(got["dx"][:, keep]).all()) and bool(torch.isfinite(got["dweight"]).all())
        assert not got["dweight"][5].any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [9, 150])
def test_rows_whose_gradients_are_zero_may_be_nan(rows, dtype):
    x, w, tokens, mask, a, b = _case(rows, 40, 300, dtype, 4, True)
    a[::3], b[::3] = 0, 0
    want = _run(x, w, tokens, mask, a, b, dtype)
    x[::3] = float("nan")
    got = _run(x, w, tokens, mask, a, b, dtype)
    assert not want["dx"][::3].any() and torch.equal(got["dx"], want["dx"]) and torch.equal(got["dweight"], want["dweight"])
