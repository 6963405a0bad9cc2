"""The smooth activations over every finite 16-bit argument, held to errors relative to their own value, the far negative
side included. Needs a B200.

Bounds. The value is the argument times a factor (the normal or logistic distribution function) that is evaluated in
binary32 through 2^x with |x| <= 126. Below that the factor leaves binary32's normal range and may be flushed to zero:
2^-126 times |z| < 88, 2^-119 absolute. x is a polynomial of at most nine roundings, constants included, each 2^-24 of it:
126 ln 2 9 2^-24 = 4.7e-5 of the factor; the rest (approximate exponential, reciprocal, a polynomial of ten terms) is a few
units of 2^-22: 2^-14 covers both. The derivative is the sum of the
factor and z times its slope, each within 2^-14 of itself. One rounding to the output type follows."""
import math

import pytest
import torch

import hgemm_reference as ref
import paper_2003_00532_b200 as dg

pytestmark = pytest.mark.gpu

TYPES = [torch.bfloat16, torch.float16]
SMOOTH = [ref.GELU, ref.GELU_TANH, ref.SILU]
ROUGH, FLUSHED = 2.0 ** -14, 2.0 ** -119


def _parts(z, act):
    """Factor and z times the factor's slope, in 64 bits without cancellation."""
    if act == ref.GELU:
        return 0.5 * torch.special.erfc(-z / math.sqrt(2)), z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act == ref.SILU:
        q = torch.sigmoid(z)
        return q, z * q * torch.sigmoid(-z)
    c = 2 * math.sqrt(2 / math.pi)
    p = c * (z + 0.044715 * z ** 3)
    q = torch.sigmoid(p)
    return q, z * q * torch.sigmoid(-p) * c * (1 + 3 * 0.044715 * z * z)


def _all(dtype):
    x = torch.arange(-32768, 32768, device="cuda", dtype=torch.int32).to(torch.int16).view(dtype)
    return x[torch.isfinite(x)].contiguous()


def _value_bound(v, dtype):
    err = ROUGH * v.abs() + FLUSHED
    return ref.rounded(v, err, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("act", SMOOTH)
def test_values(act, dtype):
    z = _all(dtype)
    z = z[z.double().abs() < 2.0 ** 60]          # (the cube of the tanh form's argument stays within 64 bits' reach)
    factor, _ = _parts(z.double(), act)
    want = z.double() * factor
    bound = _value_bound(want, dtype)
    ones = torch.ones(8, 1, dtype=dtype, device="cuda")
    D = torch.empty(z.numel(), 8, dtype=dtype, device="cuda")
    dg.hgemm_epilogue(z[:, None], ones, D, act=act, transb=True)              # tensor cores
    ref.assert_within(D, want[:, None].expand(-1, 8), bound[:, None].expand(-1, 8), "values")
    row = torch.empty(1, z.numel(), dtype=dtype, device="cuda")
    weights = torch.zeros(z.numel(), 8, dtype=dtype, device="cuda")
    weights[:, 0] = z
    dg.hgemm_epilogue(ones.t()[:, :8].contiguous(), weights, row, act=act, transb=True)       # one row
    ref.assert_within(row[0], want, bound, "values of one row")
    pair = torch.stack((z, torch.ones_like(z)), 1)
    wg, wu = (torch.tensor(w, dtype=dtype, device="cuda").expand(8, 2).contiguous() for w in ((1.0, 0.0), (0.0, 1.0)))
    H = torch.empty(z.numel(), 8, dtype=dtype, device="cuda")
    dg.hgemm_gated(pair, wg, wu, H, act=act, transw=True)
    ref.assert_within(H, want[:, None].expand(-1, 8), bound[:, None].expand(-1, 8), "gated values")
    assert dg.hgemm_last_device_status() == dg.DGEMM_OK


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("act", SMOOTH)
def test_derivatives(act, dtype):
    z = _all(dtype)
    z = z[z.double().abs() < 2.0 ** 30]
    factor, slope = _parts(z.double(), act)
    want = factor + slope
    err = ROUGH * (factor + slope.abs()) + FLUSHED * (1 + z.double().abs())
    one = torch.ones(1, 1, dtype=dtype, device="cuda")
    dD = torch.ones(z.numel(), 1, dtype=dtype, device="cuda")
    dA = torch.empty(z.numel(), 1, dtype=dtype, device="cuda")
    dg.hgemm_epilogue_bwd(z[:, None], one, dD, act=act, preact=z[:, None], dA=dA, transb=True)
    ref.assert_within(dA[:, 0], want, ref.rounded(want, err + ref.U[dtype] * want.abs() + ref.TINY[dtype], dtype), "derivative")
    # the bias gradient sums binary32 values: one row gives the derivative unrounded
    db = torch.empty(z.numel(), device="cuda")
    dg.hgemm_epilogue_bwd(one, z[:, None], dD.t().contiguous(), act=act, preact=z[None, :], dbias=db, transb=True)
    ref.assert_within(db, want, err + 2.0 ** -22 * (factor + slope.abs()) + 1e-38, "derivative in binary32")
    # gated: dX = dH U act'(G) Wg + dH act(G) Wu with dH = U = Wg = 1, Wu = 0
    dX = torch.empty(z.numel(), 1, dtype=dtype, device="cuda")
    dg.hgemm_gated_bwd(z[:, None], one, torch.zeros_like(one), z[:, None], dD, dD, act=act, dX=dX, transw=True)
    ref.assert_within(dX[:, 0], want, ref.rounded(want, err + ref.U[dtype] * want.abs() + ref.TINY[dtype], dtype), "gated derivative")
    dX2 = torch.empty(z.numel(), 1, dtype=dtype, device="cuda")
    dg.hgemm_gated_bwd(z[:, None], torch.zeros_like(one), one, z[:, None], dD, dD, act=act, dX=dX2, transw=True)
    v = z.double() * factor
    ref.assert_within(dX2[:, 0], v, ref.rounded(v, ROUGH * v.abs() + FLUSHED + ref.U[dtype] * v.abs() + ref.TINY[dtype], dtype), "gated value")
    assert dg.hgemm_last_device_status() == dg.DGEMM_OK
