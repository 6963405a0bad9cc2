"""How many bits the sums of 8-bit products keep, on the tensor cores and in the kernels for up to eight rows, and every 8-bit value as an operand of
these. Needs a B200.

A term 2^e between +2^16 and -2^16 has to be left over, exactly, when the two have cancelled, as in binary32: for every e down to -7 (2^16 + 2^-7 has 24
significant bits) if the terms lie in different instructions, whose sums are added in turn, and so if they lie in one. The outputs are powers of
two and are not rounded."""
import pytest
import torch

import paper_2003_00532_b200 as dg
import rows_reference as rr
from test_gpu_hgemm import _ok

pytestmark = pytest.mark.gpu

BF = torch.bfloat16
NAN = float("nan")


def _factors(e):
    """Two e4m3 values whose product is 2^e, -15 <= e <= 16."""
    a = max(-6, min(8, e))
    return 2.0 ** a, 2.0 ** (e - a)


def _operands(M, N, K, at, exponents):
    """Every row of A times every row of B: 2^16 + the small terms - 2^16, in this order, at the columns `at`; row m has the term of exponents[m]."""
    A, B = torch.zeros(M, K, device="cuda"), torch.zeros(N, K, device="cuda")
    first, small, last = at
    A[:, first], B[:, first] = 256.0, 256.0
    A[:, last], B[:, last] = -256.0, 256.0
    for m in range(M):
        A[m, small] = _factors(exponents[m % len(exponents)])[0]
    assert len({_factors(e)[1] for e in exponents}) == 1
    B[:, small] = _factors(exponents[0])[1]
    return A.to(rr.E4M3), B.to(rr.E4M3)


# columns of the three terms: in one instruction of 32 values; in one of 16; in two halves of one; in one k-block; in different k-blocks; in
# different warps' shares of a token's sum and in one warp's (512 apart)
PLACES = [(0, 1, 2), (3, 9, 15), (0, 20, 31), (0, 40, 100), (5, 300, 900), (0, 512, 1024), (17, 530, 1040), (1024, 512, 0), (1100, 70, 900)]


@pytest.mark.parametrize("at", PLACES)
@pytest.mark.parametrize("M,N,K", [(1, 40, 1200), (3, 40, 1201), (8, 300, 1200), (9, 300, 1200), (64, 256, 1216), (300, 520, 1201), (700, 1000, 1200)])
def test_small_terms_between_large_ones(M, N, K, at):
    for exponents in ([-6, -5, -4, -3, -2, -1, 0, 1, 2, 5, 8], [-7]):
        A, B = _operands(M, N, K, at, exponents)
        want = torch.tensor([2.0 ** exponents[m % len(exponents)] for m in range(M)], device="cuda")[:, None]
        D = torch.full((M, N), NAN, dtype=BF, device="cuda")
        dg.qgemm_epilogue(A, B, D)
        assert torch.equal(D.float(), want.expand(M, N))
        G, U, H = (torch.full((M, N), NAN, dtype=BF, device="cuda") for _ in range(3))
        dg.qgemm_gated(A, B, B, H, act=dg.HGEMM_ACT_NONE, gate=G, up=U)
        assert torch.equal(G.float(), want.expand(M, N)) and torch.equal(U, G) and torch.equal(H.float(), (want * want).expand(M, N))
    _ok()


@pytest.mark.parametrize("M,N", [(40, 300), (200, 260)])
def test_small_terms_in_a_sum_that_is_cut_into_parts(M, N):
    """A long sum over few tiles: parts are added in binary32, too."""
    K = 9000
    for at in ((0, 4000, 8999), (8999, 10, 5000), (4000, 4001, 4002)):
        A, B = _operands(M, N, K, at, [-6, -3, 0])
        want = torch.tensor([2.0 ** [-6, -3, 0][m % 3] for m in range(M)], device="cuda")[:, None]
        D = torch.full((M, N), NAN, dtype=BF, device="cuda")
        dg.qgemm_epilogue(A, B, D)
        assert torch.equal(D.float(), want.expand(M, N))
    _ok()


@pytest.mark.parametrize("M", [1, 2, 5, 8, 9])
def test_every_8_bit_value_beside_few_rows(M):
    """All 256 codes as weights, and, a few at a time, as activations."""
    codes = torch.arange(256, dtype=torch.uint8, device="cuda").view(rr.E4M3)
    want = codes.float().bfloat16()
    nan = torch.isnan(want)
    W = torch.zeros(256, 160, dtype=rr.E4M3, device="cuda")
    W[:, 77] = codes
    X = torch.zeros(M, 160, device="cuda")
    X[:, 77] = torch.tensor([1.0, -2.0, 0.5, 4.0, -1.0, 2.0, 1.0, 0.25, 1.0], device="cuda")[:M]
    X8 = X.to(rr.E4M3)
    D, G, U, H = (torch.full((M, 256), 3.0, dtype=BF, device="cuda") for _ in range(4))
    dg.qgemm_epilogue(X8, W, D)
    dg.qgemm_gated(X8, W, W, H, act=dg.HGEMM_ACT_NONE, gate=G, up=U)
    for out in (D, G, U):
        assert torch.equal(torch.isnan(out), nan.expand(M, 256))
        assert torch.equal(out[:, ~nan].float(), want[~nan].float() * X[:, 77:78])
    for first in range(0, 256, M):
        part = codes[first:first + M]
        A = torch.zeros(len(part), 160, dtype=rr.E4M3, device="cuda")
        A[:, 77] = part
        B = torch.ones(40, 160, device="cuda").to(rr.E4M3)
        D = torch.full((len(part), 40), 3.0, dtype=BF, device="cuda")
        dg.qgemm_epilogue(A, B, D)
        v = part.float().bfloat16()[:, None].expand_as(D)
        assert torch.equal(torch.isnan(D), torch.isnan(v)) and torch.equal(D[~torch.isnan(v)], v[~torch.isnan(v)])
    _ok()
