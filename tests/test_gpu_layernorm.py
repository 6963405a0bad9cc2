"""Layer norm, forward and backward, against plain 64-bit forms (bounds: ``hgemm_reference``). Needs a B200."""
import pytest
import torch

import hgemm_reference as ref
import paper_2003_00532_b200 as dg
from test_gpu_hgemm import _gen, _out, _padding_intact, _place

pytestmark = pytest.mark.gpu

TYPES = [torch.bfloat16, torch.float16, torch.float32]


def _rows(g, rows, cols, dtype, pad=0, offset=0):
    x = torch.randn(rows, cols, device="cuda", generator=g) * (0.5 + 2 * torch.rand(rows, 1, device="cuda", generator=g))
    return _place((x + torch.randn(rows, 1, device="cuda", generator=g)).to(dtype), pad, offset)


def _vector(g, n, dtype, mid):
    return (torch.randn(n, device="cuda", generator=g) * 0.3 + mid).to(dtype)


def _forward(rows, cols, dtype, eps=1e-5, affine=True, stats=True, seed=0, pad=0, offset=0):
    g = _gen(seed)
    X, Y = _rows(g, rows, cols, dtype, pad, offset), _out(rows, cols, dtype, pad, offset)
    gamma, beta = (_vector(g, cols, dtype, 1.0), _vector(g, cols, dtype, 0.0)) if affine else (None, None)
    mean, rstd = (torch.full((rows,), float("nan"), device="cuda") for _ in range(2)) if stats else (None, None)
    dg.layernorm_fwd(X, gamma, beta, Y, eps=eps, mean=mean, rstd=rstd)
    y, ye, m, me, r, re = ref.norm(X, gamma, beta, eps)
    assert _padding_intact(Y)
    ref.assert_within(Y, y, ye, "Y")
    if stats:
        ref.assert_within(mean, m, me + 2.0 ** -23 * m.abs(), "mean")
        ref.assert_within(rstd, r, re, "rstd")


def _backward(rows, cols, dtype, affine=True, seed=0, pad=0, offset=0, want=("dx", "dgamma", "dbeta")):
    g = _gen(seed)
    X, dY = _rows(g, rows, cols, dtype, pad, offset), _rows(g, rows, cols, dtype, pad, offset)
    gamma = _vector(g, cols, dtype, 1.0) if affine else None
    mean = X.double().mean(1).float()
    rstd = (X.double().var(1, unbiased=False) + 1e-5).rsqrt().float()
    out = {"dx": _out(rows, cols, dtype, pad, offset), "dgamma": torch.full((cols,), float("nan"), device="cuda"),
           "dbeta": torch.full((cols,), float("nan"), device="cuda")}
    names = {"dx": "dX"}
    dg.layernorm_bwd(X, gamma, mean, rstd, dY, **{names.get(k, k): v for k, v in out.items() if k in want})
    for name, (v, bound) in ref.norm_grad(X, gamma, mean, rstd, dY).items():
        if name not in want:
            assert bool(torch.isnan(out[name]).all())
            continue
        if name == "dx":
            assert _padding_intact(out[name])
        ref.assert_within(out[name], v, bound, name)


SIZES = [(1, 1), (3, 1), (1, 2), (5, 7), (9, 31), (8, 32), (17, 33), (7, 100), (1, 256), (33, 257), (20, 512), (12, 1000), (3, 1025),
         (1, 4096), (300, 1537), (10, 4096), (5, 5001), (4, 8192), (2, 8200), (3, 16384), (2, 16391), (1, 40000)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", SIZES)
def test_forward(size, dtype):
    _forward(*size, dtype, seed=sum(size))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", SIZES + [(2000, 64), (700, 4096), (4097, 200)])
def test_backward(size, dtype):
    _backward(*size, dtype, seed=sum(size))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pad,offset", [(8, 0), (3, 0), (0, 1), (5, 3)])
@pytest.mark.parametrize("size", [(9, 100), (40, 1000), (6, 5000), (2, 20000)])
def test_strides_and_alignment(size, pad, offset, dtype):
    _forward(*size, dtype, seed=pad, pad=pad, offset=offset)
    _backward(*size, dtype, seed=pad, pad=pad, offset=offset)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", [(5, 300), (6, 3000), (2, 20000)])
def test_without_parameters_and_statistics(size, dtype):
    _forward(*size, dtype, affine=False, stats=False)
    _backward(*size, dtype, affine=False)


@pytest.mark.parametrize("want", [("dx",), ("dgamma",), ("dbeta",), ("dgamma", "dbeta"), ("dx", "dbeta")])
@pytest.mark.parametrize("size", [(50, 200), (50, 3000), (9, 20000)])
def test_optional_gradients(size, want):
    _backward(*size, torch.bfloat16, want=want)


@pytest.mark.parametrize("cols", [7, 600, 3000, 20000])
def test_large_mean_keeps_the_variance(cols):
    """Rows with a mean 1000 times their deviation: the variance must not come from a difference of large sums."""
    g = _gen(2)
    X = torch.randn(11, cols, device="cuda", generator=g) + 1000.0
    Y, rstd = torch.empty_like(X), torch.empty(11, device="cuda")
    dg.layernorm_fwd(X, None, None, Y, rstd=rstd)
    y, ye, _, _, r, re = ref.norm(X, None, None, 1e-5)
    ref.assert_within(rstd, r, re, "rstd")
    ref.assert_within(Y, y, ye, "Y")


def test_constant_rows_and_zero_epsilon():
    X = torch.full((3, 500), 2.5, device="cuda", dtype=torch.bfloat16)
    Y, rstd = torch.empty_like(X), torch.empty(3, device="cuda")
    dg.layernorm_fwd(X, None, None, Y, eps=1e-5, rstd=rstd)
    assert bool((Y == 0).all()) and torch.allclose(rstd, torch.full_like(rstd, 1e-5 ** -0.5), rtol=1e-6)
    _forward(40, 300, torch.float32, eps=0.0)


def test_nan_and_infinity_stay_in_their_row():
    g = _gen(5)
    X = _rows(g, 20, 700, torch.float16)
    X[3, 9], X[11, 650] = float("nan"), float("inf")
    Y = _out(20, 700, torch.float16)
    dg.layernorm_fwd(X, None, None, Y)
    bad = torch.zeros(20, dtype=torch.bool, device="cuda")
    bad[3], bad[11] = True, True
    assert bool(torch.isnan(Y[bad]).all()) and bool(torch.isfinite(Y[~bad]).all())


def test_same_bits_every_time():
    g = _gen(6)
    X, dY = _rows(g, 3000, 1000, torch.bfloat16), _rows(g, 3000, 1000, torch.bfloat16)
    mean, rstd = X.float().mean(1), X.float().var(1, unbiased=False).add(1e-5).rsqrt()
    runs = []
    for _ in range(5):
        dX, a, b = torch.empty_like(X), torch.empty(1000, device="cuda"), torch.empty(1000, device="cuda")
        dg.layernorm_bwd(X, None, mean, rstd, dY, dX=dX, dgamma=a, dbeta=b)
        runs.append((dX, a, b))
    for r in runs[1:]:
        assert all(torch.equal(x, y) for x, y in zip(r, runs[0]))


def test_gradient_agrees_with_differences():
    g = _gen(7)
    X, dY = _rows(g, 6, 90, torch.float32), _rows(g, 6, 90, torch.float32)
    gamma, beta = _vector(g, 90, torch.float32, 1.0), _vector(g, 90, torch.float32, 0.0)
    Y, mean, rstd = torch.empty_like(X), torch.empty(6, device="cuda"), torch.empty(6, device="cuda")
    dg.layernorm_fwd(X, gamma, beta, Y, mean=mean, rstd=rstd)
    dX, dga, dbe = torch.empty(6, 90, device="cuda"), torch.empty(90, device="cuda"), torch.empty(90, device="cuda")
    dg.layernorm_bwd(X, gamma, mean, rstd, dY, dX=dX, dgamma=dga, dbeta=dbe)
    E = [torch.randn(*s, device="cuda", generator=g).double() for s in ((6, 90), (90,), (90,))]

    def f(s):
        return float((dY.double() * ref.norm(X.double() + s * E[0], gamma.double() + s * E[1], beta.double() + s * E[2], 1e-5)[0]).sum())

    h = 1e-5
    slope = (f(h) - f(-h)) / (2 * h)
    parts = [(dX.double() * E[0]), (dga.double() * E[1]), (dbe.double() * E[2])]
    # every gradient is known to 2^-18 or so of its size in binary32; the differences to h^2
    assert abs(sum(float(p.sum()) for p in parts) - slope) <= 2.0 ** -18 * sum(float(p.abs().sum()) for p in parts) + 1e-5


def test_empty_and_refusals():
    bf = torch.bfloat16
    dg.layernorm_fwd(torch.zeros(0, 8, dtype=bf, device="cuda"), None, None, torch.zeros(0, 8, dtype=bf, device="cuda"))
    dg.layernorm_fwd(torch.zeros(4, 0, dtype=bf, device="cuda"), None, None, torch.zeros(4, 0, dtype=bf, device="cuda"))
    a, b = torch.full((8,), float("nan"), device="cuda"), torch.full((8,), float("nan"), device="cuda")
    none = torch.zeros(0, device="cuda")
    dg.layernorm_bwd(torch.zeros(0, 8, dtype=bf, device="cuda"), None, none, none, torch.zeros(0, 8, dtype=bf, device="cuda"), dgamma=a, dbeta=b)
    assert bool((a == 0).all()) and bool((b == 0).all())
    X, Y = torch.zeros(4, 8, dtype=bf, device="cuda"), torch.zeros(4, 8, dtype=bf, device="cuda")
    with pytest.raises(dg.DgemmError):
        dg.layernorm_fwd(X, None, None, X)           # overlapping
    with pytest.raises(dg.DgemmError):
        dg.layernorm_fwd(X, None, None, Y, eps=-1.0)
    with pytest.raises(dg.DgemmError):
        dg.layernorm_fwd(X, None, None, Y, eps=float("nan"))
    with pytest.raises(dg.DgemmError):
        dg.layernorm_bwd(X, None, None, None, Y, dX=torch.zeros_like(X))
    with pytest.raises(TypeError):
        dg.layernorm_fwd(X, torch.ones(8, device="cuda"), None, Y)
    with pytest.raises(ValueError):
        dg.layernorm_fwd(X, torch.ones(7, device="cuda", dtype=bf), None, Y)
    with pytest.raises(TypeError):
        dg.layernorm_fwd(X.double(), None, None, Y)
