"""The activations' derivatives before any rounding to 16 bits: the bias gradient of one row, for every finite 16-bit argument,
held to the bound that ``hgemm_reference`` gives for it (2^-20 of dD and five units of 2^-23 of the value). Needs a B200."""
import pytest
import torch

import hgemm_reference as ref
import paper_2003_00532_b200 as dg
from test_gpu_gelu_tail import _all

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("act", ref.ACTS)
def test_slope_of_one_row(act, dtype):
    z = _all(dtype)
    z = z[z.double().abs() < 2.0 ** 30]
    Z, dD = z[None, :].contiguous(), torch.ones(1, z.numel(), dtype=dtype, device="cuda")
    A, B = torch.ones(1, 1, dtype=dtype, device="cuda"), torch.ones(z.numel(), 1, dtype=dtype, device="cuda")
    db = torch.empty(z.numel(), device="cuda")
    dg.hgemm_epilogue_bwd(A, B, dD, act=act, preact=Z, dbias=db, transb=True)
    want, bound = ref.linear_grad(A, B, Z, act, dD, False, True)["dbias"]
    ref.assert_within(db, want, bound, "slope")
