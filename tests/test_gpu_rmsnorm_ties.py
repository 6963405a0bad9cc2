"""16-bit rows brought to 8 bits are the nearest e4m3 values to 448 x / max|x|, bit for bit, ties to even: such quotients lie half-way between two
values quite often (both have few digits). Needs a B200.

The quotient in 64 bits: 448 x is exact, the division rounds once and gives a tie exactly; any other quotient is away from a tie by at least
2^-16 of itself (x and max have 11 bits at the most, a tie 5)."""
import pytest
import torch

import paper_2003_00532_b200 as dg
import rows_reference as rr
import test_gpu_rmsnorm as base
from test_gpu_hgemm import _gen

pytestmark = pytest.mark.gpu


def _nearest(X):
    v = X.double() * 448 / X.double().abs().amax(1, keepdim=True).clamp_min(rr.LEAST)
    step = 2 * rr.half_step(v)
    return v, torch.round(v / step) * step


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("size", [(2000, 300), (500, 1000), (300, 4089), (2088, 4096), (600, 8192), (100, 12000), (30, 20000), (30, 20001)])
def test_nearest_value_and_ties_to_even(size, dtype):
    X = base.rows_of(_gen(sum(size)), *size, dtype)
    (Q, _), scale = base.eight_out(*size), base.f32(size[0])
    dg.quantize_rows_e4m3(X, Q, scale)
    v, want = _nearest(X)
    ties = (v - want).abs() == rr.half_step(v)
    assert int(ties.sum()) > 0
    assert torch.equal(Q.double(), want)
    assert torch.equal(torch.signbit(Q.float()), torch.signbit(X))


@pytest.mark.parametrize("dtype,exponents", [(torch.bfloat16, (-91, 0, 100, 118)), (torch.float16, (-5, 0, 6))])
def test_every_largest_value(dtype, exponents):
    """Rows whose largest value runs over every significand, from small ones to the type's largest; all ties among the values that the type has."""
    bits = 8 if dtype is torch.bfloat16 else 11
    top = (1 + torch.arange(2 ** (bits - 1), device="cuda").double() / 2 ** (bits - 1))[:, None]
    codes = torch.arange(127, dtype=torch.uint8, device="cuda").view(rr.E4M3).double()
    mid = (codes[1:] + codes[:-1]) / 2
    for e in exponents:
        X = torch.cat([top, -(top * mid / 448), top * mid / 448, -0.0 * top], 1) * 2.0 ** e
        X = X.to(dtype)
        X[:, 0] = (top[:, 0] * 2.0 ** e).to(dtype)
        (Q, _), scale = base.eight_out(*X.shape), base.f32(X.shape[0])
        dg.quantize_rows_e4m3(X, Q, scale)
        v, want = _nearest(X)
        assert int(((v - want).abs() == rr.half_step(v)).sum()) > 100
        assert torch.equal(Q.double(), want) and torch.equal(torch.signbit(Q.float()), torch.signbit(X))
