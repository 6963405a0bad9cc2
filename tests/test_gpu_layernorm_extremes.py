"""Layer norm's gradients where (0 - mean) rstd, which no column has, leaves binary32's range: it must not reach the row's sums.
Needs a B200.

Bound: the rows are constant, so xh is exactly 0 and dx = rstd (w - mean(w)): the sum errs by 256 2^-24 of the mean of |w| as in
``hgemm_reference``, the rest by a few roundings."""
import pytest
import torch

import hgemm_reference as ref
import paper_2003_00532_b200 as dg
from test_gpu_hgemm import _gen, _out, _place

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("cols", [1, 5, 8, 33, 100, 1001, 4000, 5001, 9000, 20000])
@pytest.mark.parametrize("pad", [0, 1])
def test_constant_rows_of_large_values(cols, dtype, pad):
    g = _gen(cols)
    value = torch.tensor(1e37, dtype=dtype, device="cuda")
    X = _place(value.expand(6, cols).contiguous(), pad)
    dY = _place(torch.randn(6, cols, device="cuda", generator=g).to(dtype), pad)
    gamma = (torch.randn(cols, device="cuda", generator=g) * 0.3 + 1).to(dtype)
    mean, rstd = value.float().expand(6).contiguous(), torch.full((6,), 1e-5 ** -0.5, device="cuda")
    dX, dga, dbe = _out(6, cols, dtype, pad), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    dg.layernorm_bwd(X, gamma, mean, rstd, dY, dX=dX, dgamma=dga, dbeta=dbe)
    w, r = dY.double() * gamma.double(), rstd.double()[:, None]
    s = w.mean(1, keepdim=True)
    want = r * (w - s)
    err = r * (256 * 2.0 ** -24 * w.abs().mean(1, keepdim=True) + 2.0 ** -22 * (w.abs() + s.abs()))
    ref.assert_within(dX, want, ref.rounded(want, err, dtype), "dx")
    assert bool((dga == 0).all())
    ref.assert_within(dbe, dY.double().sum(0), 22 * 2.0 ** -23 * dY.double().abs().sum(0) + 1e-38, "dbeta")
