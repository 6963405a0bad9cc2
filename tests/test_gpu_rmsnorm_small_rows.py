"""RMS norm to 8 bits where a row is zero or very small beside an eps that lets rstd become large: the scale is that of 2^-100 / 448 then, and
rstd times its reciprocal leaves binary32's range although q does not. Needs a B200.

Bounds of ``rows_reference``: y within VALUE of its size, q within half a step of e4m3 and that. What a product s gamma below binary32's
smallest normal value loses (2^-150) may move q by 2^-30 at the most, which is what the half step is widened by (2^-10 times 2^-20)."""
import pytest
import torch

import paper_2003_00532_b200 as dg
import rows_reference as rr
import test_gpu_rmsnorm as base
import test_gpu_rmsnorm_extremes as many
from test_gpu_hgemm import _gen

pytestmark = pytest.mark.gpu

SHAPES = base.SHAPES + many.SHAPES
EPS = [1e-5, 1e-8, 2.7e-12, 1e-12, 1e-20, 1e-27, 1e-35]


def _binary32(x):
    return float(torch.tensor(x, dtype=torch.float32))


def _rows(shape, dtype, sizes, seed):
    """Rows of these sizes in turn, their signs and values drawn."""
    size = torch.tensor(sizes, dtype=torch.float64, device="cuda").repeat((shape[0] + len(sizes) - 1) // len(sizes))[:shape[0], None]
    return (torch.randn(*shape, device="cuda", generator=_gen(seed)).double() * size).to(dtype)


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dtype", base.TYPES)
def test_zero_rows_are_zero_for_every_eps(shape, dtype):
    X = _rows(shape, dtype, [1.0, 0.0, 0.0], 1)
    gamma = base.vector_of(_gen(2), shape[1], dtype)
    least = float(torch.tensor(2.0 ** -100, dtype=torch.float32) / 448)
    for eps in EPS:
        (Q, _), scale, r = base.eight_out(*shape), base.f32(shape[0]), base.f32(shape[0])
        dg.rmsnorm_fwd_e4m3(X, gamma, Q, scale, eps=eps, rstd=r)
        zero = (X == 0).all(1)
        assert int(zero.sum()) > 0 and bool((Q[zero].float() == 0).all()) and bool((scale[zero] == least).all()), eps
        want = _binary32(eps) ** -0.5
        assert bool(((r[zero].double() - want).abs() <= rr.VALUE * want).all()), eps
        rr.assert_eight(Q, scale, rr.rms(X, None, gamma, _binary32(eps))[1])


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("res", [False, True])
def test_small_rows_keep_their_values(shape, dtype, res):
    """Ordinary, small, hardly normal and subnormal rows, with and without a residual (s + s: exact) and with the sum kept."""
    X = _rows(shape, dtype, [1e-37, 1.0, 1e-30, 2.0 ** -119, 1e-20, 1e-39], 3)
    gamma = base.vector_of(_gen(4), shape[1], dtype)
    for eps in EPS:
        y = rr.rms(X, X if res else None, gamma, _binary32(eps))[1]
        (Q, _), scale, S = base.eight_out(*shape), base.f32(shape[0]), torch.empty_like(X)
        dg.rmsnorm_fwd_e4m3(X, gamma, Q, scale, eps=eps, residual=X.clone() if res else None, sum=S if res else None)
        rr.assert_eight(Q, scale, y)
        assert not res or torch.equal(S, X + X)


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("s,gamma,eps", [(2.0 ** -44, 2.0 ** -100, 0.0), (2.0 ** -70, 2.0 ** -60, 2.0 ** -66), (2.0 ** 55, 2.0 ** 75, 0.0), (1.0, 2.0 ** -125, 1e-5)])
def test_weights_far_from_one(shape, dtype, s, gamma, eps):
    """s gamma below or above binary32's normal range, y inside it."""
    X = _rows(shape, dtype, [s], 5)
    w = (base.vector_of(_gen(6), shape[1], torch.float32).double() * gamma).to(dtype)
    (Q, _), scale = base.eight_out(*shape), base.f32(shape[0])
    dg.rmsnorm_fwd_e4m3(X, w, Q, scale, eps=eps)
    rr.assert_eight(Q, scale, rr.rms(X, None, w, eps)[1])
