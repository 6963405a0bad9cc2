"""RMS norm's rows out of binary32's range, zero rows, NaN and infinities where there are many rows, aligned and not: the kernels that take rows
through shared memory. Cases and bounds of test_gpu_rmsnorm. Needs a B200."""
import pytest
import torch

import hgemm_reference as ref
import paper_2003_00532_b200 as dg
import rows_reference as rr
import test_gpu_rmsnorm as base
from test_gpu_hgemm import _gen

pytestmark = pytest.mark.gpu

# (one block of 256 or 512 threads, 32 values per thread, single values; odd: misaligned alike)
SHAPES = [(1100, 1000), (4000, 1001), (700, 4096), (1000, 4089), (700, 5120), (800, 5001), (2400, 2600), (1300, 8192), (500, 8191), (400, 9000), (500, 9001), (9000, 100)]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dtype,size", [(torch.float32, 1e30), (torch.bfloat16, 1e25), (torch.bfloat16, 1e38), (torch.float32, 2e-43), (torch.bfloat16, 1e-35)])
def test_rows_whose_squares_leave_the_range(shape, dtype, size):
    base.test_rows_whose_squares_leave_the_range(shape, dtype, size)


@pytest.mark.parametrize("shape", SHAPES)
def test_some_rows_out_of_range_beside_a_residual(shape):
    """Ordinary rows and rows that are scaled first, in turn, with a residual of their size: sum, norm and 8 bits."""
    rows, cols = shape
    g = _gen(cols)
    size = torch.tensor([1.0, 2.0 ** 70, 2.0 ** -70, 1.0, 2.0 ** 100], dtype=torch.float64, device="cuda").repeat((rows + 4) // 5)[:rows, None]
    X, R = ((torch.randn(rows, cols, device="cuda", generator=g).double() * size).bfloat16() for _ in range(2))
    gamma = base.vector_of(g, cols, torch.bfloat16)
    s, y, rstd = rr.rms(X, R, gamma, 0.0)
    S, Y, r = torch.empty_like(X), torch.empty_like(X), base.f32(rows)
    dg.rmsnorm_fwd(X, gamma, Y, eps=0.0, residual=R, sum=S, rstd=r)
    ref.assert_within(S, s, rr.sum_bound(s, torch.bfloat16), "S")
    ref.assert_within(Y, y, rr.value_bound(y, torch.bfloat16), "Y")
    ref.assert_within(r, rstd, rr.VALUE * rstd, "rstd")
    (Q, _), scale = base.eight_out(rows, cols), base.f32(rows)
    dg.rmsnorm_fwd_e4m3(X, gamma, Q, scale, eps=0.0, residual=R, sum=S)
    rr.assert_eight(Q, scale, y)


@pytest.mark.parametrize("shape", SHAPES)
def test_small_and_zero_rows_nan_and_infinity(shape):
    base.test_small_rows_under_an_eps(shape)
    base.test_zero_rows(shape)
    base.test_nan_and_infinity_stay_in_their_row(shape)


@pytest.mark.parametrize("size", [(2400, 1000), (700, 5120), (700, 5001), (400, 9000), (500, 9001), (9000, 99)])
def test_same_bits_every_time(size):
    g = _gen(6)
    S, dY, dS = (base.rows_of(g, *size, torch.bfloat16) for _ in range(3))
    rstd = (S.float().square().mean(1) + 1e-5).rsqrt()
    runs = []
    for _ in range(4):
        dX, a = torch.empty_like(S), base.f32(size[1])
        dg.rmsnorm_bwd(S, None, rstd, dY, dsum=dS, dX=dX, dgamma=a)
        runs.append((dX, a))
    for r in runs[1:]:
        assert all(torch.equal(x, y) for x, y in zip(r, runs[0]))
