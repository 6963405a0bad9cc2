"""The factor 448 / max|y| by which rows are brought to 8 bits, over all exponents of binary32 and for random significands: a row of every e4m3
value times t has to come out as these values again, with scale = max / 448 as the division gives it. Needs a B200.

Each value c t is off by 2^-24 of itself, the factor and the product with it by as much again (under the norm by at most VALUE): far less than the
half step, 2^-5 of c or more, that c is away from the next border."""
import pytest
import torch

import paper_2003_00532_b200 as dg
import rows_reference as rr
import test_gpu_rmsnorm as base
from test_gpu_hgemm import _gen

pytestmark = pytest.mark.gpu


def _rows(cols, exponents, significands, dtype):
    codes = torch.arange(127, dtype=torch.uint8, device="cuda").view(rr.E4M3).double()     # 0 .. 448
    codes = torch.cat([codes.flip(0), -codes]).repeat(cols // 254 + 1)[:cols]
    t = torch.exp2(torch.arange(*exponents, device="cuda").double())[:, None] * significands
    t = t.flatten()[:, None]
    return (codes * t).to(dtype), codes, t


@pytest.mark.parametrize("cols", [254, 1000, 4096, 9001, 20000])
def test_every_exponent(cols):
    significands = torch.cat([torch.ones(1, device="cuda"), 1 + torch.rand(4, device="cuda", generator=_gen(cols))]).double()
    X, codes, t = _rows(cols, (-108, 118), significands, torch.float32)
    (Q, _), scale = base.eight_out(*X.shape), base.f32(X.shape[0])
    dg.quantize_rows_e4m3(X, Q, scale)
    assert torch.equal(Q.double(), codes.expand_as(Q.double()))
    assert torch.equal(scale, X.abs().amax(1) / torch.full_like(scale, 448))
    dg.rmsnorm_fwd_e4m3(X, None, Q, scale, eps=0.0)
    assert torch.equal(Q.double(), codes.expand_as(Q.double()))
    rr.assert_eight(Q, scale, rr.rms(X, None, None, 0.0)[1])


@pytest.mark.parametrize("dtype,exponents", [(torch.bfloat16, (-108, 118)), (torch.float16, (-14, 7))])
@pytest.mark.parametrize("cols", [254, 1000, 4089, 9001, 20000])
def test_every_exponent_in_16_bits(dtype, exponents, cols):
    X, codes, t = _rows(cols, exponents, torch.ones(1, dtype=torch.float64, device="cuda"), dtype)
    X = X.repeat(3, 1)     # (enough rows for the kernels for many)
    (Q, _), scale = base.eight_out(*X.shape), base.f32(X.shape[0])
    dg.quantize_rows_e4m3(X, Q, scale)
    assert torch.equal(Q.double(), codes.expand_as(Q.double())) and torch.equal(scale, t[:, 0].float().repeat(3))
    dg.rmsnorm_fwd_e4m3(X, None, Q, scale, eps=0.0)
    assert torch.equal(Q.double(), codes.expand_as(Q.double()))


def test_rows_that_are_smaller_than_the_least():
    """From 2^-100 down all rows have one scale; a zero, an infinity and a NaN."""
    t = torch.exp2(torch.arange(-149, -99, device="cuda").double())[:, None]
    X = (t * torch.tensor([1.0, -0.5, 0.25, 0.0], dtype=torch.float64, device="cuda")).float()
    (Q, _), scale = base.eight_out(*X.shape), base.f32(X.shape[0])
    dg.quantize_rows_e4m3(X, Q, scale)
    least = torch.tensor(2.0 ** -100, device="cuda") / torch.tensor(448.0, device="cuda")
    assert bool((scale == least).all())
    rr.assert_eight(Q, scale, X.double(), value=0.0)
    X = torch.tensor([[0.0, 0.0], [float("inf"), 1.0], [float("nan"), 1.0]], device="cuda")
    (Q, _), scale = base.eight_out(3, 2), base.f32(3)
    dg.quantize_rows_e4m3(X, Q, scale)
    assert bool((Q[0].float() == 0).all()) and float(scale[0]) == float(least)
    assert float(scale[1]) == float("inf") and bool(torch.isnan(Q[1, 0].float())) and float(Q[1, 1].float()) == 0.0
    assert bool(torch.isnan(scale[2])) and bool(torch.isnan(Q[2].float()).all())
