"""The planes of fp32 operands, on the CPU: what three hold, what six of their nine products leave out, and that the bounds of planes_ref.py tell three planes
from two."""
import torch

import planes_ref as ref


def _values(n, seed):
    gen = torch.Generator().manual_seed(seed)
    v = torch.randn(n, generator=gen)
    hard = torch.tensor([1.0078124, 1.0 + 2.0 ** -8, 1.0 + 2.0 ** -8 - 2.0 ** -23, 1.99609375, 2.0 - 2.0 ** -23, 1.0 + 2.0 ** -8 + 2.0 ** -16 - 2.0 ** -23])
    return torch.cat([v, hard, -hard])


def test_three_planes_hold_every_bit():
    v = torch.cat([_values(100000, 1), torch.tensor([3.4028235e38, -3.4028235e38, 3.3961776e38, 1e-30, 2.0 ** -109])])
    assert torch.equal(sum(p.double() for p in ref.planes(v)), v.double())
    assert all(bool(torch.isfinite(p).all()) for p in ref.planes(v))


def test_six_products_leave_out_half_a_step_of_fp32():
    # planes are 2^-8 of a value and, of one that is not a power of two further, 2^-17: 2^-8 2^-17 2 + 2^-34
    a, b = _values(300000, 2), _values(300000, 3).flip(0)
    p, q = ([x.double() for x in ref.planes(v)] for v in (a, b))
    six = p[0] * q[0] + p[0] * q[1] + p[1] * q[0] + p[1] * q[1] + p[0] * q[2] + p[2] * q[0]
    rel = (six - a.double() * b.double()) / (a.double() * b.double())
    assert float(rel.abs().max()) <= 2.0 ** -24 * (1 + 2.0 ** -9)
    assert abs(float(rel.mean())) <= 2.0 ** -30          # 300000 of both signs, 2^-26 each


def test_the_bounds_tell_three_planes_from_two():
    gen = torch.Generator().manual_seed(4)
    for n in (100, 200, 300):
        a, b = torch.randn(200, n, generator=gen), torch.randn(n, 150, generator=gen)
        two = sum(ref.planes(a, 2)).double() @ sum(ref.planes(b, 2)).double()
        assert ref.off(two, a.double() @ b.double()) >= ref.TWO >= 4 * ref.product_off(n)
