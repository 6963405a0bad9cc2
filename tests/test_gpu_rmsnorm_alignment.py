"""RMS norm on rows that are not 16-byte aligned: all matrices misaligned alike (every shift, rows shorter than a vector, more rows than are
on their way at once, leading dimensions whose shifts repeat sooner) and each in its own way. Bounds as in test_gpu_rmsnorm. Needs a B200."""
import pytest
import torch

import hgemm_reference as ref
import paper_2003_00532_b200 as dg
import rows_reference as rr
from test_gpu_hgemm import _gen, _out, _padding_intact
from test_gpu_rmsnorm import TYPES, backward, eight_out, eight_padding_intact, f32, forward, forward8, rows8, rows_of, vector_of

pytestmark = pytest.mark.gpu


def everything(rows, cols, dtype, **at):
    forward(rows, cols, dtype, seed=rows, **at)
    forward(rows, cols, dtype, res=False, keep=False, seed=rows, **at)
    forward8(rows, cols, dtype, seed=rows, **at)
    rows8(rows, cols, dtype, seed=rows, **at)
    backward(rows, cols, dtype, seed=rows, **at)
    backward(rows, cols, dtype, ds=False, affine=False, seed=rows, **at)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("offset", range(8))
@pytest.mark.parametrize("pad", [1, 4])
def test_every_shift(offset, pad, dtype):
    """1024 + pad: rows one value apart, or shifts that repeat after two rows; a short and a long matrix."""
    everything(5, 1024, dtype, pad=pad, offset=offset)
    everything(1201, 1024, dtype, pad=pad, offset=offset)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", list(range(1, 18)) + [31, 249, 255, 257])
def test_short_rows(cols, dtype):
    everything(9001, cols, dtype)
    everything(37, cols, dtype, pad=2, offset=3)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", [(3001, 505), (2500, 513), (5000, 1001), (2600, 2047), (2600, 4089), (1300, 4097), (900, 8185), (900, 8186), (700, 9001), (400, 16377),
                                  (400, 16378), (5, 16379), (1, 16383), (1, 4097)])
def test_lengths(size, dtype):
    everything(*size, dtype)
    everything(*size, dtype, pad=2, offset=1)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", [(900, 200), (700, 1001), (300, 5000), (40, 12001)])
def test_every_matrix_in_its_own_way(size, dtype):
    rows, cols = size
    g = _gen(cols)
    X, R, dY = rows_of(g, rows, cols, dtype, 1, 0), rows_of(g, rows, cols, dtype, 2, 3), rows_of(g, rows, cols, dtype, 0, 5)
    S, Y, dX = _out(rows, cols, dtype, 3, 1), _out(rows, cols, dtype, 5, 2), _out(rows, cols, dtype, 4, 7)
    gamma, rstd = vector_of(g, cols, dtype), f32(rows)
    s, y, r = rr.rms(X, R, gamma, 1e-5)
    dg.rmsnorm_fwd(X, gamma, Y, residual=R, sum=S, rstd=rstd)
    ref.assert_within(Y, y, rr.value_bound(y, dtype), "Y")
    ref.assert_within(S, s, rr.sum_bound(s, dtype), "S")
    ref.assert_within(rstd, r, rr.VALUE * r, "rstd")
    (Q, whole), scale = eight_out(rows, cols, 3, 2), f32(rows)
    dg.rmsnorm_fwd_e4m3(X, gamma, Q, scale, residual=R)
    rr.assert_eight(Q, scale, y)
    expected, dga = rr.rms_grad(S, gamma, rstd, dY, R), f32(cols)
    dg.rmsnorm_bwd(S, gamma, rstd, dY, dsum=R, dX=dX, dgamma=dga)
    ref.assert_within(dX, *expected["dX"], "dX")
    ref.assert_within(dga, *expected["dgamma"], "dgamma")
    assert all(_padding_intact(t) for t in (S, Y, dX)) and eight_padding_intact(Q, whole, 3, 2)


@pytest.mark.parametrize("dtype", TYPES)
def test_weights_at_any_address(dtype):
    """Aligned rows with a weight that is not."""
    for rows, cols in ((5, 1024), (1201, 1024), (700, 4096), (300, 12000)):
        g = _gen(cols)
        X, dY, gamma = rows_of(g, rows, cols, dtype), rows_of(g, rows, cols, dtype), vector_of(g, cols + 1, dtype)[1:]
        Y, rstd, dX, dga = torch.empty_like(X), f32(rows), torch.empty_like(X), f32(cols)
        _, y, _ = rr.rms(X, None, gamma, 1e-5)
        dg.rmsnorm_fwd(X, gamma, Y, rstd=rstd)
        ref.assert_within(Y, y, rr.value_bound(y, dtype), "Y")
        dg.rmsnorm_bwd(X, gamma, rstd, dY, dX=dX, dgamma=dga)
        expected = rr.rms_grad(X, gamma, rstd, dY, None)
        ref.assert_within(dX, *expected["dX"], "dX")
        ref.assert_within(dga, *expected["dgamma"], "dgamma")


@pytest.mark.parametrize("cols", [33, 1001, 4097, 9001])
@pytest.mark.parametrize("dtype", TYPES)
def test_an_infinite_statistic_stays_in_its_row(cols, dtype):
    """What lies before and beyond an unaligned row must not make it NaN where rstd is infinite in its neighbour."""
    rows = 2001
    S, dY = torch.randn(rows, cols, device="cuda", generator=_gen(1)).to(dtype), torch.randn(rows, cols, device="cuda", generator=_gen(2)).to(dtype)
    rstd = torch.ones(rows, device="cuda")
    rstd[7::13] = float("inf")
    S[7::13], dY[7::13] = 1, 0
    dX, dga = torch.empty_like(S), f32(cols)
    dg.rmsnorm_bwd(S, None, rstd, dY, dX=dX)
    bad = torch.isinf(rstd)
    assert bool(torch.isfinite(dX[~bad]).all()) and bool(torch.isnan(dX[bad]).all())
