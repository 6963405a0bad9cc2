"""RMS norm under weights so large or small that s gamma leaves binary32's normal range where y = s rstd gamma lies inside it, in every kernel
shape. Needs a B200. Bounds of ``rows_reference``: y within VALUE of its size, then one rounding."""
import pytest
import torch

import hgemm_reference as ref
import paper_2003_00532_b200 as dg
import rows_reference as rr
import test_gpu_rmsnorm as base
import test_gpu_rmsnorm_extremes as many
from test_gpu_hgemm import _gen

pytestmark = pytest.mark.gpu

SHAPES = base.SHAPES + many.SHAPES


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("res", [False, True])
@pytest.mark.parametrize("size,gamma,eps", [(2.0 ** 55, 2.0 ** 75, 0.0), (1e15, 1e24, 1e-5), (2.0 ** 53, 2.0 ** 100, 1e-5), (2.0 ** 70, 2.0 ** 100, 0.0),
                                            (2.0 ** -44, 2.0 ** -100, 0.0), (1e-12, 1e-30, 0.0), (2.0 ** -70, 2.0 ** -90, 0.0), (1.0, 2.0 ** 120, 1e-5)])
def test_y_is_right_where_s_gamma_is_out_of_range(shape, dtype, res, size, gamma, eps):
    g = _gen(shape[1])
    X, R = ((torch.randn(*shape, device="cuda", generator=g).double() * size).to(dtype) for _ in range(2))
    w = (base.vector_of(g, shape[1], torch.float32).double() * gamma).to(dtype)
    s, y, rstd = rr.rms(X, R if res else None, w, float(torch.tensor(eps, dtype=torch.float32)))
    Y, S, r = torch.empty_like(X), torch.empty_like(X), base.f32(shape[0])
    dg.rmsnorm_fwd(X, w, Y, eps=eps, residual=R if res else None, sum=S if res else None, rstd=r)
    ref.assert_within(Y, y, rr.value_bound(y, dtype), "Y")
    ref.assert_within(r, rstd, rr.VALUE * rstd, "rstd")
    if res:
        ref.assert_within(S, s, rr.sum_bound(s, dtype), "S")
