"""What a gated pair keeps of its forward pass is what it computed: gradients of bf16 plans are those of g and u in fp32, rounded as operands alone."""
import pytest
import torch

import more_operators_ref as ref
from paper_2304_07741_amd import binding as B
from paper_2304_07741_amd import harness

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", [B.CANVAS_GATED_SIGMOID, B.CANVAS_GATED_SILU, B.CANVAS_GATED_GELU], ids=["sigmoid", "silu", "gelu"])
@pytest.mark.parametrize("rows,width", [(1, 5000), (40, 5000), (300, 5003)])
def test_gates_are_kept_whole(rows, width, kind):
    # One row has a gradient, and its first feature is 1: that column of dWg and dWu is dg and du, rounded to bf16 once.  Off by half a step of bf16, of the power of two below the
    # value, and by what fp32 makes of g, u, act and slope (32 u of each factor's largest terms).  Gates and values have more bits than bf16 or 20 bits hold.
    features = 16
    gen = torch.Generator().manual_seed(rows)
    x = torch.randn(rows, features, generator=gen) * 2.0 ** -6
    x[0, 0] = 1
    x, wg, wu = x.bfloat16(), torch.randn(width, features, generator=gen).bfloat16(), torch.randn(width, features, generator=gen).bfloat16()
    dy = torch.zeros(rows, width, dtype=torch.bfloat16)
    dy[0] = 1
    t = [v.cuda() for v in (x, wg, wu, dy)]
    r = harness.GatedRunner(rows, features, width, "bf16", kind)
    r.forward(*t[:3])
    out = r.backward(*t)
    g, u = (t[0][0].double() @ w.double().T for w in t[1:3])
    a, da = ref.act(kind, g)
    off = 32 * ref.U
    for name, want, large in (("dw_up", a, a.abs() + 1.13 * g.abs()), ("dw_gate", u * da, (u.abs() + 3) * (1 + g.abs()))):
        got = out[name][:, 0].double()
        half = torch.exp2(torch.floor(torch.log2(want.abs().clamp_min(1e-30) * (1 + 2.0 ** -20))) - 8)
        over = (got - want).abs() - half - off * (large + 1)
        assert float(over.max()) <= 0, (name, float(over.max()), int((over > 0).sum()))
    r.close()
