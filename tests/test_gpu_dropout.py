"""Dropout with the residual's addition, forward and backward, against its definition (``rows_reference``). Needs a B200."""
import pytest
import torch

import hgemm_reference as ref
import paper_2003_00532_b200 as dg
import rows_reference as rr
from test_gpu_hgemm import _gen, _out, _padding_intact, _place

pytestmark = pytest.mark.gpu

TYPES = [torch.bfloat16, torch.float16, torch.float32]
SEED, OFFSET = 0x9E3779B97F4A7C15, 2 ** 40 + 17


def _matrix(g, rows, cols, dtype, pad=0, offset=0):
    x = torch.randn(rows, cols, device="cuda", generator=g)
    x[x == 0] = 1
    return _place(x.to(dtype), pad, offset)


def _case(rows, cols, dtype, p=0.3, res=True, pad=0, offset=0, place=None, seed=SEED, use=OFFSET):
    g = _gen(rows + cols)
    X = _matrix(g, rows, cols, dtype, pad, offset)
    R = _matrix(g, rows, cols, dtype, pad, offset) if res else None
    y, bound, keep = rr.dropout(X, R, p, seed, use)
    d, dbound, _ = rr.dropout(X, None, p, seed, use)
    dX = _out(rows, cols, dtype, pad, offset)
    dg.dropout_bwd(X, dX, p, seed, use)
    Y = {"X": X, "R": R, None: _out(rows, cols, dtype, pad, offset)}[place]
    dg.dropout_fwd(X, Y, p, seed, use, residual=R)
    assert _padding_intact(Y) and _padding_intact(dX)
    ref.assert_within(Y, y, bound, "Y")
    ref.assert_within(dX, d, dbound, "dX")
    if p < 1:
        assert torch.equal(dX != 0, keep)        # bit for bit the same mask
    assert bool((dX[~keep] == 0).all())


SIZES = [(1, 1), (1, 3), (5, 4), (3, 7), (2, 8), (9, 31), (17, 64), (1, 4096), (33, 257), (300, 1537), (4097, 12), (1000, 2048), (3, 40001), (70000, 5)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", SIZES)
def test_forward_and_backward(size, dtype):
    _case(*size, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pad,offset", [(8, 0), (3, 0), (0, 1), (5, 3), (4, 4)])
@pytest.mark.parametrize("size", [(9, 100), (200, 1001), (31, 4096)])
def test_strides_and_alignment(size, pad, offset, dtype):
    """The mask is the same at any address and leading dimension."""
    _case(*size, dtype, pad=pad, offset=offset)


@pytest.mark.parametrize("p", [0.0, 1.0, 0.5, 1e-3, 0.999, 2.0 ** -32, 1 - 2.0 ** -20, 1 - 2.0 ** -34])
def test_probabilities(p):
    for dtype in (torch.bfloat16, torch.float32):
        _case(100, 333, dtype, p=p)


@pytest.mark.parametrize("res", [False, True])
@pytest.mark.parametrize("pad", [0, 3])
def test_in_place(pad, res):
    for dtype in TYPES:
        _case(300, 1000, dtype, res=res, pad=pad, place="X")
        if res:
            _case(300, 1000, dtype, pad=pad, place="R")


@pytest.mark.parametrize("seed,use", [(0, 0), (1, 0), (2 ** 32, 0), (2 ** 64 - 1, 2 ** 64 - 1), (5, 2 ** 32), (-1, -3)])
def test_seeds_and_offsets(seed, use):
    _case(40, 100, torch.float16, seed=seed, use=use) if seed >= 0 else None
    a, b = (torch.empty(40, 100, dtype=torch.float16, device="cuda") for _ in range(2))
    X = torch.ones_like(a)
    dg.dropout_fwd(X, a, 0.5, seed, use)
    dg.dropout_fwd(X, b, 0.5, seed % 2 ** 64, use % 2 ** 64)
    assert torch.equal(a, b)
    dg.dropout_fwd(X, b, 0.5, seed, use + 1)
    assert not torch.equal(a, b)


def test_share_that_is_kept():
    """4 million values: the share of ones is p within five standard deviations, over rows, columns and words of a block alike."""
    X = torch.ones(2000, 2000, device="cuda")
    Y = torch.empty_like(X)
    for p in (0.1, 0.5, 0.9):
        dg.dropout_fwd(X, Y, p, 1234, 5)
        kept = (Y != 0).double()
        sd = (p * (1 - p)) ** 0.5
        assert abs(float(kept.mean()) - (1 - p)) < 5 * sd / 2000
        for axis in (0, 1):
            assert float((kept.mean(axis) - (1 - p)).abs().max()) < 6 * sd / 2000 ** 0.5
        for j in range(4):
            assert abs(float(kept[:, j::4].mean()) - (1 - p)) < 5 * sd / 1000


def test_what_is_dropped_counts_as_zero():
    X = torch.full((50, 203), float("nan"), device="cuda")
    X[:, ::2] = float("inf")
    R = torch.randn(50, 203, device="cuda", generator=_gen(1))
    Y = torch.empty_like(X)
    dg.dropout_fwd(X, Y, 0.4, 3, 4, residual=R)
    keep = rr.words(50, 203, 3, 4, "cuda") >= int(0.4 * 2 ** 32 + 0.5)
    assert torch.equal(Y[~keep], R[~keep]) and not bool(torch.isfinite(Y[keep]).any())
    dg.dropout_fwd(X, Y, 1.0, 3, 4)
    assert bool((Y == 0).all())


def test_step_on_the_device_and_replays():
    """A captured call: the counter on the device gives every replay a mask of its own, forward and backward the same one."""
    X, Y, D = (torch.ones(64, 300, dtype=torch.bfloat16, device="cuda") for _ in range(3))
    step = torch.zeros(1, dtype=torch.int64, device="cuda")

    def call():
        dg.dropout_fwd(X, Y, 0.5, 11, 100, step=step)
        dg.dropout_bwd(X, D, 0.5, 11, 100, step=step)
        step.add_(1)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        call()
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            call()
    for i in range(1, 5):
        graph.replay()
        torch.cuda.synchronize()
        keep = rr.words(64, 300, 11, 100 + i, "cuda") >= 2 ** 31
        assert torch.equal(Y != 0, keep) and torch.equal(D != 0, keep)
    step.fill_(-101)                                   # offset + step wraps below zero
    dg.dropout_fwd(X, Y, 0.5, 11, 100, step=step)
    assert torch.equal(Y != 0, rr.words(64, 300, 11, 2 ** 64 - 1, "cuda") >= 2 ** 31)


def test_another_stream():
    s = torch.cuda.Stream()
    X = torch.randn(500, 1000, device="cuda", generator=_gen(1))
    Y = torch.empty_like(X)
    torch.cuda.synchronize()
    dg.dropout_fwd(X, Y, 0.2, 1, 2, stream=s)
    s.synchronize()
    y, bound, _ = rr.dropout(X, None, 0.2, 1, 2)
    ref.assert_within(Y, y, bound, "Y")


def test_gradient_agrees_with_differences():
    """y is linear in x for a fixed mask."""
    g = _gen(3)
    X, E, dY, R = (torch.randn(20, 301, device="cuda", generator=g) for _ in range(4))
    Y, Z, dX = torch.empty_like(X), torch.empty_like(X), torch.empty_like(X)
    dg.dropout_fwd(X, Y, 0.3, 8, 9, residual=R)
    dg.dropout_fwd(X + E, Z, 0.3, 8, 9, residual=R)
    dg.dropout_bwd(dY, dX, 0.3, 8, 9)
    want = float((dX.double() * E.double()).sum())
    got = float((dY.double() * (Z.double() - Y.double())).sum())
    # Y and Z are off by 2^-22 of their terms, X + E by 2^-24
    assert abs(got - want) <= 2.0 ** -21 * float((dY.double().abs() * (X.abs() + E.abs() + R.abs()).double()).sum()) / 0.7


def test_rows_beyond_2_to_the_31_values():
    """A wide leading dimension and a late part of a long matrix: positions in 64 bits."""
    rows, ld = 66000, 32777
    X = torch.empty((rows - 1) * ld + 9, dtype=torch.float16, device="cuda").as_strided((rows, 9), (ld, 1))
    X.fill_(1)
    Y = torch.empty((rows - 1) * ld + 9, dtype=torch.float16, device="cuda").as_strided((rows, 9), (ld, 1))
    dg.dropout_fwd(X, Y, 0.5, 1, 2)
    assert torch.equal(Y != 0, rr.words(rows, 9, 1, 2, "cuda") >= 2 ** 31)
    del X, Y
    rows, cols = 2 ** 19 + 3, 4100
    X = torch.ones(rows, cols, dtype=torch.float16, device="cuda")
    Y = torch.empty_like(X)
    dg.dropout_fwd(X, Y, 0.5, 1, 2)
    for r in (0, 2 ** 18, rows - 50):
        assert torch.equal(Y[r:r + 50] != 0, rr.words(50, cols, 1, 2, "cuda", first_row=r) >= 2 ** 31)


def test_empty_and_refusals():
    e = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device="cuda")   # noqa: E731
    dg.dropout_fwd(e(0, 8), e(0, 8), 0.5, 1)
    dg.dropout_fwd(e(8, 0), e(8, 0), 0.5, 1)
    X = e(4, 8)
    for p in (-0.5, 1.01, float("nan")):
        with pytest.raises(dg.DgemmError):
            dg.dropout_fwd(X, e(4, 8), p, 1)
    with pytest.raises(TypeError):
        dg.dropout_fwd(X, e(4, 8), 0.5, 1.5)
    with pytest.raises(TypeError):
        dg.dropout_fwd(X, e(4, 8), 0.5, 1, step=torch.zeros(1, device="cuda"))
    with pytest.raises(ValueError):
        dg.dropout_fwd(X, e(4, 8), 0.5, 1, step=torch.zeros(1, dtype=torch.int64))
    with pytest.raises(ValueError):
        dg.dropout_fwd(X, e(4, 9), 0.5, 1)
    with pytest.raises(TypeError):
        dg.dropout_fwd(X.double(), X.double(), 0.5, 1)
