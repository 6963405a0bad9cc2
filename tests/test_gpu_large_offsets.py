"""Matrices whose last elements lie more than 2^31 elements behind the first: wide leading dimensions and large outputs, in every
operator. Needs a B200 (30 GB of its memory). Integer data where sums are exact; the bounds of ``hgemm_reference`` elsewhere."""
import pytest
import torch

import hgemm_reference as ref
import paper_2003_00532_b200 as dg
from test_gpu_hgemm import _gen, _ok

pytestmark = pytest.mark.gpu

BF = torch.bfloat16
ROWS, LD = 66000, 32776          # 2.16e9 elements; rows of 16-byte vectors
ODD = 32777                      # rows of any alignment


def _wide(rows, cols, ld, dtype=BF):
    """An uninitialised view of `rows` rows `ld` elements apart."""
    return torch.empty((rows - 1) * ld + cols, dtype=dtype, device="cuda").as_strided((rows, cols), (ld, 1))


def _ints(g, rows, cols, ld, dtype=BF):
    x = _wide(rows, cols, ld, dtype)
    x.copy_(torch.randint(-3, 4, (rows, cols), device="cuda", generator=g))
    return x


@pytest.mark.parametrize("ld", [LD, ODD])
def test_product_and_gradients(ld):
    g = _gen(1)
    M, N, K = ROWS, 72, 40
    A, B = _ints(g, M, K, ld), _ints(g, N, K, K)
    D, Z = _wide(M, N, ld), _wide(M, N, ld)
    dg.hgemm_epilogue(A, B, D, act=dg.HGEMM_ACT_RELU, preact=Z, transb=True)
    want = A.double() @ B.double().t()
    assert torch.equal(Z, want.to(BF)) and torch.equal(D, want.clamp_min(0).to(BF))
    dD = D
    dD.copy_(torch.randint(-3, 4, (M, N), device="cuda", generator=g))
    dA, dB, db = _wide(M, K, ld), torch.empty(N, K, dtype=BF, device="cuda"), torch.empty(N, device="cuda")
    dg.hgemm_epilogue_bwd(A, B, dD, act=dg.HGEMM_ACT_RELU, preact=Z, dA=dA, dB=dB, dbias=db, transb=True)
    dz = dD.double() * (Z.double() > 0)
    assert torch.equal(dA, (dz @ B.double()).to(BF)) and torch.equal(dB, (dz.t() @ A.double()).to(BF)) and torch.equal(db.double(), dz.sum(0))
    _ok()


@pytest.mark.parametrize("ld", [LD, ODD])
def test_weights_of_a_token(ld):
    """One and two rows against weights stored N x K over a wide leading dimension, and transposed operands."""
    g = _gen(2)
    W, x = _ints(g, ROWS, 48, ld), _ints(g, 2, 48, 48)
    want = (x.double() @ W.double().t()).to(BF)
    for rows in (1, 2):
        D = torch.empty(rows, ROWS, dtype=BF, device="cuda")
        dg.hgemm_epilogue(x[:rows], W, D, transb=True)
        assert torch.equal(D, want[:rows])
        H = torch.empty(rows, ROWS, dtype=BF, device="cuda")
        dg.hgemm_gated(x[:rows], W, W, H, act=dg.HGEMM_ACT_NONE, transw=True)
        assert torch.equal(H, (x[:rows].double() @ W.double().t()).square().to(BF))
    # contraction over the distant rows
    A, D = _ints(g, ROWS, 24, ld), torch.empty(24, 48, dtype=BF, device="cuda")
    dg.hgemm_epilogue(A, W, D, transa=True)
    assert torch.equal(D, (A.double().t() @ W.double()).to(BF))
    _ok()


@pytest.mark.parametrize("ld", [LD, ODD])
def test_gated_and_gradients(ld):
    g = _gen(3)
    M, F, K = ROWS, 72, 40
    X, Wg, Wu = _ints(g, M, K, ld), _ints(g, F, K, K), _ints(g, F, K, K)
    H, G, U = (_wide(M, F, ld) for _ in range(3))
    dg.hgemm_gated(X, Wg, Wu, H, act=dg.HGEMM_ACT_RELU, gate=G, up=U, transw=True)
    zg, zu = X.double() @ Wg.double().t(), X.double() @ Wu.double().t()
    assert torch.equal(G, zg.to(BF)) and torch.equal(U, zu.to(BF)) and torch.equal(H, (zg.clamp_min(0) * zu).to(BF))
    for t in (H, G, U):
        t.copy_(torch.randint(-3, 4, (M, F), device="cuda", generator=g))
    dX, dWg, dWu = _wide(M, K, ld), torch.empty(F, K, dtype=BF, device="cuda"), torch.empty(F, K, dtype=BF, device="cuda")
    dg.hgemm_gated_bwd(X, Wg, Wu, G, U, H, act=dg.HGEMM_ACT_RELU, dX=dX, dWg=dWg, dWu=dWu, transw=True)
    a, dh = G.double(), H.double()
    dgate, dup = dh * U.double() * (a > 0), dh * a.clamp_min(0)
    assert torch.equal(dX, (dgate @ Wg.double() + dup @ Wu.double()).to(BF))
    assert torch.equal(dWg, (dgate.t() @ X.double()).to(BF)) and torch.equal(dWu, (dup.t() @ X.double()).to(BF))
    _ok()


def test_output_of_more_than_32_bits():
    """M N beyond 2^31, dense: every tile's place, forward and in the element-wise gradient."""
    g = _gen(4)
    M, N, K = 47000, 46000, 24
    A, B = _ints(g, M, K, K), _ints(g, N, K, K)
    D = torch.empty(M, N, dtype=BF, device="cuda")
    dg.hgemm_epilogue(A, B, D, transb=True)
    for r in range(0, M, 4700):
        assert torch.equal(D[r:r + 4700], (A[r:r + 4700].float() @ B.float().t()).to(BF))     # (sums of at most 216: exact)
    db = torch.empty(N, device="cuda")
    dA = torch.empty(M, K, dtype=BF, device="cuda")
    dg.hgemm_epilogue_bwd(A, B, D, act=dg.HGEMM_ACT_RELU, preact=D, dA=dA, dbias=db, transb=True)
    sums = torch.zeros(N, dtype=torch.float64, device="cuda")
    for r in range(0, M, 4700):
        dz = D[r:r + 4700].double().clamp_min(0)
        sums += dz.sum(0)
        v, size = dz @ B.double(), dz @ B.double().abs()
        ref.assert_within(dA[r:r + 4700], v, ref.rounded(v, ref.sum_error(N, size), BF), "dA")
    assert torch.equal(db.double(), sums)
    _ok()


@pytest.mark.parametrize("ld", [LD, ODD])
@pytest.mark.parametrize("cols", [100, 1200])
def test_layernorm(cols, ld):
    g = _gen(5)
    X, Y, dY, dX = (_wide(ROWS, cols, ld) for _ in range(4))
    for t in (X, dY):
        t.copy_(torch.randn(ROWS, cols, device="cuda", generator=g))
    gamma = (torch.randn(cols, device="cuda", generator=g) * 0.3 + 1).to(BF)
    mean, rstd = torch.empty(ROWS, device="cuda"), torch.empty(ROWS, device="cuda")
    dga, dbe = torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    dg.layernorm_fwd(X, gamma, None, Y, mean=mean, rstd=rstd)
    dg.layernorm_bwd(X, gamma, mean, rstd, dY, dX=dX, dgamma=dga, dbeta=dbe)
    y, ye, m, me, r, re = ref.norm(X, gamma, None, 1e-5)
    ref.assert_within(Y, y, ye, "Y")
    ref.assert_within(mean, m, me + 2.0 ** -23 * m.abs(), "mean")
    ref.assert_within(rstd, r, re, "rstd")
    for got, (name, (v, bound)) in zip((dX, dga, dbe), ref.norm_grad(X, gamma, mean, rstd, dY).items()):
        ref.assert_within(got, v, bound, name)
