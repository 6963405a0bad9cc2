"""Products of one to eight rows of 8-bit operands on both sides of every border between the kernel for few rows and the one for many (columns per
SM, length of the sum), and the former on weights of more than 2^31 bytes. Needs a B200. Bounds of ``rows_reference``; integer data exact."""
import pytest
import torch

import hgemm_reference as ref
import paper_2003_00532_b200 as dg
import rows_reference as rr
import test_gpu_qgemm as base
from test_gpu_hgemm import _gen

pytestmark = pytest.mark.gpu

SMS = 148


@pytest.mark.parametrize("M", [1, 2, 8, 9])
@pytest.mark.parametrize("N", [32 * SMS, 32 * SMS + 1, 64 * SMS, 64 * SMS + 1])
@pytest.mark.parametrize("K", [1024, 2032, 2048, 4080, 4096])
def test_borders(M, N, K):
    base._linear(M, N, K, torch.bfloat16, integer=True, seed=M, save=False)
    base._linear(M, N, K, torch.float16, act=ref.SILU, seed=M, res=False)
    base._gated(M, N, K, torch.bfloat16, ref.NONE, integer=True, seed=M)
    base._gated(M, N, K, torch.float16, ref.SILU, seed=M, save=False)


@pytest.mark.parametrize("M", [1, 3, 8])
def test_gated_weights_of_more_than_2_to_the_31_bytes(M):
    F, K = 70001, 32768
    W = torch.zeros(F, K, dtype=torch.uint8, device="cuda").view(rr.E4M3)
    W[-5:] = (torch.randn(5, K, device="cuda", generator=_gen(1)) * 0.5).to(rr.E4M3)
    X = (torch.randn(M, K, device="cuda", generator=_gen(2)) * 0.5).to(rr.E4M3)
    H, G, U = (torch.empty(M, F, dtype=torch.bfloat16, device="cuda") for _ in range(3))
    dg.qgemm_gated(X, W, W, H, act=dg.HGEMM_ACT_SILU, gate=G, up=U)
    want = rr.gated8(X, W[-5:], W[-5:], None, None, None, ref.SILU, torch.bfloat16)
    for name, out in (("H", H), ("G", G), ("U", U)):
        ref.assert_within(out[:, -5:], *want[name], name)
        assert bool((out[:, :-5] == 0).all())


@pytest.mark.parametrize("M", [1, 4])
def test_weights_of_more_than_2_to_the_31_bytes(M):
    """Few, long rows: the kernel for few rows takes them."""
    N, K = 64, 2 ** 25 + 2 ** 24 + 80
    B = torch.zeros(N, K, dtype=torch.uint8, device="cuda").view(rr.E4M3)
    A = torch.zeros(M, K, dtype=torch.uint8, device="cuda").view(rr.E4M3)
    g = _gen(3)
    for at in (0, K // 2, K - 1000):
        B[:, at:at + 1000] = (torch.randn(N, 1000, device="cuda", generator=g) * 0.5).to(rr.E4M3)
        A[:, at:at + 1000] = (torch.randn(M, 1000, device="cuda", generator=g) * 0.5).to(rr.E4M3)
    D = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    dg.qgemm_epilogue(A, B, D)
    part = torch.cat([torch.arange(at, at + 1000, device="cuda") for at in (0, K // 2, K - 1000)])
    d, bound, _, _ = rr.linear8(A.view(torch.uint8)[:, part].view(rr.E4M3), B.view(torch.uint8)[:, part].view(rr.E4M3), None, None, None, ref.NONE, None, torch.bfloat16)
    ref.assert_within(D, d, bound, "D")
