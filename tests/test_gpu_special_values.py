"""NaN and infinities in the gated projections, in every gradient and in layer norm's gradients: they reach the rows and columns
whose sums they enter and no others. Needs a B200.

Everything else is compared bit for bit with the same call without them (an entry that a NaN or an infinity replaces is 0 there,
and what it enters is left out of the comparison)."""
import pytest
import torch

import hgemm_reference as ref
import paper_2003_00532_b200 as dg
from test_gpu_hgemm import TYPES, _draw, _gen, _ok, _out

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")


def _same_except(got, want, rows=(), cols=(), what="", open_rows=()):
    """``rows`` and ``cols`` are lost; ``open_rows`` change and may be finite."""
    keep = torch.ones(got.shape, dtype=torch.bool, device="cuda")
    for r in (*rows, *open_rows):
        keep[r] = False
    for c in cols:
        keep[..., c] = False
    assert bool(torch.isfinite(want).all()), what
    assert torch.equal(got[keep], want[keep]), what + ": a value outside the affected rows and columns changed"
    for r in rows:
        assert not bool(torch.isfinite(got[r]).all()), what
    for c in cols:
        assert not bool(torch.isfinite(got[..., c]).all()), what


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("act", ref.ACTS)
@pytest.mark.parametrize("shape", [(2, 140, 72), (150, 140, 70), (40, 300, 3000)])
def test_product(shape, act, dtype):
    M, N, K = shape
    g = _gen(act)
    A, B = _draw(g, M, K, dtype), _draw(g, N, K, dtype, K ** -0.5)
    A[M - 1, 5], B[130, 0] = 0.0, 0.0
    outs = []
    for bad in (False, True):
        if bad:
            A[M - 1, 5], B[130, 0] = NAN, INF
        D, Z = _out(M, N, dtype), _out(M, N, dtype)
        dg.hgemm_epilogue(A, B, D, act=act, preact=Z, transb=True)
        outs.append((D, Z))
    _ok()
    _same_except(outs[1][1], outs[0][1], [M - 1], [130], "Z")
    keep = torch.ones(M, N, dtype=torch.bool, device="cuda")
    keep[M - 1], keep[:, 130] = False, False
    assert torch.equal(outs[1][0][keep], outs[0][0][keep])
    assert bool(torch.isnan(outs[1][0][M - 1]).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("act", ref.ACTS)
@pytest.mark.parametrize("shape", [(1, 140, 72), (150, 140, 70), (40, 300, 3000)])
def test_gated(shape, act, dtype):
    M, F, K = shape
    g = _gen(act)
    X, Wg, Wu = _draw(g, M, K, dtype), _draw(g, F, K, dtype, K ** -0.5), _draw(g, F, K, dtype, K ** -0.5)
    Wg[7, 3], Wu[131, 2] = 0.0, 0.0
    outs = []
    for bad in (False, True):
        if bad:
            Wg[7, 3], Wu[131, 2] = NAN, NAN
        H, G, U = _out(M, F, dtype), _out(M, F, dtype), _out(M, F, dtype)
        dg.hgemm_gated(X, Wg, Wu, H, act=act, gate=G, up=U, transw=True)
        outs.append((H, G, U))
    _ok()
    for got, want, cols, name in zip(outs[1], outs[0], ((7, 131), (7,), (131,)), "HGU"):
        _same_except(got, want, (), cols, name)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("act", ref.ACTS)
def test_product_gradients(act, dtype):
    M, N, K = 150, 200, 72
    g = _gen(act)
    A, B = _draw(g, M, K, dtype), _draw(g, N, K, dtype, K ** -0.5)
    dD, Z = _draw(g, M, N, dtype, 0.3), _draw(g, M, N, dtype)
    dD[3, 5], Z[77, 130], A[9, 11], B[33, 17] = 0.0, 1.0, 0.0, 0.0
    dD[77, 130] = 0.0
    outs = []
    for bad in (False, True):
        if bad:
            dD[3, 5], A[9, 11], B[33, 17] = INF, NAN, NAN
            Z[77, 130] = NAN          # enters its dZ through the derivative (ReLU's of NaN is 0, and none has no derivative)
        out = {"dA": _out(M, K, dtype), "dB": _out(N, K, dtype), "dbias": torch.full((N,), NAN, device="cuda")}
        dg.hgemm_epilogue_bwd(A, B, dD, act=act, preact=Z if act != ref.NONE else None, transb=True, **out)
        outs.append(out)
    _ok()
    through_z = act not in (ref.NONE, ref.RELU)
    # dD[3, 5] is infinite (or 0 times infinity where ReLU is flat)
    _same_except(outs[1]["dA"], outs[0]["dA"], [3] + [77] * through_z, [17], "dA")
    _same_except(outs[1]["dB"], outs[0]["dB"], [5] + [130] * through_z, [11], "dB")
    _same_except(outs[1]["dbias"], outs[0]["dbias"], [5] + [130] * through_z, [], "dbias")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("act", ref.ACTS)
def test_gated_gradients(act, dtype):
    M, F, K = 150, 200, 72
    g = _gen(act)
    X, Wg, Wu = _draw(g, M, K, dtype), _draw(g, F, K, dtype, K ** -0.5), _draw(g, F, K, dtype, K ** -0.5)
    G, U, dH = _draw(g, M, F, dtype), _draw(g, M, F, dtype), _draw(g, M, F, dtype, 0.3)
    G[3, 5], X[9, 11], Wu[33, 17], U[77, 130] = 1.5, 0.0, 0.0, 0.0
    outs = []
    for bad in (False, True):
        if bad:
            G[3, 5], X[9, 11], Wu[33, 17], U[77, 130] = NAN, NAN, NAN, INF
        out = {"dX": _out(M, K, dtype), "dWg": _out(F, K, dtype), "dWu": _out(F, K, dtype)}
        dg.hgemm_gated_bwd(X, Wg, Wu, G, U, dH, act=act, transw=True, **out)
        outs.append(out)
    _ok()
    # with G at 77, 130 positive or not, U there enters dG alone
    _same_except(outs[1]["dX"], outs[0]["dX"], [3, 77], [17], "dX")
    # (without activation dG does not depend on G; ReLU's derivative at NaN is 0 and takes the term of row 5 out)
    _same_except(outs[1]["dWg"], outs[0]["dWg"], [130] + [5] * (act not in (ref.NONE, ref.RELU)), [11], "dWg", [5] * (act == ref.RELU))
    _same_except(outs[1]["dWu"], outs[0]["dWu"], [5], [11], "dWu")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("cols", [5, 100, 1001, 3000, 9000, 20000])
def test_layernorm_gradients(cols, dtype):
    g = _gen(cols)
    X, dY = _draw(g, 40, cols, dtype), _draw(g, 40, cols, dtype)
    mean = X.float().mean(1)
    rstd = (X.float().var(1, unbiased=False) + 1e-5).rsqrt()
    X[3, 2], dY[17, 4], dY[20, cols - 1] = 0.0, 0.0, 0.0
    outs = []
    for bad in (False, True):
        if bad:
            X[3, 2], dY[17, 4], dY[20, cols - 1] = NAN, INF, NAN
        dX, dga, dbe = _out(40, cols, dtype), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
        dg.layernorm_bwd(X, None, mean, rstd, dY, dX=dX, dgamma=dga, dbeta=dbe)
        outs.append((dX, dga, dbe))
    _same_except(outs[1][0], outs[0][0], [3, 17, 20], [], "dX")
    for i, cols_hit, name in ((1, sorted({2, 4, cols - 1}), "dgamma"), (2, sorted({4, cols - 1}), "dbeta")):
        _same_except(outs[1][i], outs[0][i], cols_hit, [], name)
