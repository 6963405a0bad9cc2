"""RMS norm with the residual's addition, forward, in 8 bits and backward, against plain 64-bit forms (bounds: ``rows_reference``).
Needs a B200."""
import pytest
import torch

import hgemm_reference as ref
import paper_2003_00532_b200 as dg
import rows_reference as rr
from test_gpu_hgemm import _gen, _out, _padding_intact, _place

pytestmark = pytest.mark.gpu

TYPES = [torch.bfloat16, torch.float16, torch.float32]
INF, NAN = float("inf"), float("nan")


def rows_of(g, rows, cols, dtype, pad=0, offset=0):
    x = torch.randn(rows, cols, device="cuda", generator=g) * (0.5 + 2 * torch.rand(rows, 1, device="cuda", generator=g))
    return _place(x.to(dtype), pad, offset)


def vector_of(g, n, dtype, mid=1.0):
    return (torch.randn(n, device="cuda", generator=g) * 0.3 + mid).to(dtype)


def f32(n):
    return torch.full((n,), NAN, device="cuda")


def eight_out(rows, cols, pad=0, offset=0):
    """A matrix of 8-bit values in a wider buffer of bytes 0x55."""
    ld = cols + pad
    whole = torch.full((rows * ld + offset + 16,), 0x55, dtype=torch.uint8, device="cuda")
    return whole[offset:offset + rows * ld].view(rows, ld)[:, :cols].view(rr.E4M3), whole


def eight_padding_intact(Q, whole, pad, offset):
    rows, cols = Q.shape
    ld = cols + pad
    body = whole[offset:offset + rows * ld].view(rows, ld)
    return bool((whole[:offset] == 0x55).all() and (whole[offset + rows * ld:] == 0x55).all() and (body[:, cols:] == 0x55).all())


def forward(rows, cols, dtype, res=True, affine=True, keep=True, stats=True, in_place=None, eps=1e-5, seed=0, pad=0, offset=0):
    g = _gen(seed)
    X, Y = rows_of(g, rows, cols, dtype, pad, offset), _out(rows, cols, dtype, pad, offset)
    R = rows_of(g, rows, cols, dtype, pad, offset) if res else None
    gamma = vector_of(g, cols, dtype) if affine else None
    s, y, rstd = rr.rms(X, R, gamma, eps)
    S = {"X": X, "R": R, None: _out(rows, cols, dtype, pad, offset) if keep else None}[in_place]
    r = f32(rows) if stats else None
    dg.rmsnorm_fwd(X, gamma, Y, eps=eps, residual=R, sum=S, rstd=r)
    assert _padding_intact(Y) and (S is None or _padding_intact(S))
    ref.assert_within(Y, y, rr.value_bound(y, dtype), "Y")
    if S is not None:
        ref.assert_within(S, s, rr.sum_bound(s, dtype), "S")
    if stats:
        ref.assert_within(r, rstd, rr.VALUE * rstd, "rstd")


def forward8(rows, cols, dtype, res=True, affine=True, keep=True, in_place=None, seed=0, pad=0, offset=0, qpad=None, qoffset=None):
    g = _gen(seed)
    qpad, qoffset = pad if qpad is None else qpad, offset if qoffset is None else qoffset
    X = rows_of(g, rows, cols, dtype, pad, offset)
    R = rows_of(g, rows, cols, dtype, pad, offset) if res else None
    gamma = vector_of(g, cols, dtype) if affine else None
    s, y, rstd = rr.rms(X, R, gamma, 1e-5)
    S = {"X": X, "R": R, None: _out(rows, cols, dtype, pad, offset) if keep else None}[in_place]
    (Q, whole), scale, r = eight_out(rows, cols, qpad, qoffset), f32(rows), f32(rows)
    dg.rmsnorm_fwd_e4m3(X, gamma, Q, scale, residual=R, sum=S, rstd=r)
    assert eight_padding_intact(Q, whole, qpad, qoffset) and (S is None or _padding_intact(S))
    rr.assert_eight(Q, scale, y)
    ref.assert_within(r, rstd, rr.VALUE * rstd, "rstd")
    if S is not None:
        ref.assert_within(S, s, rr.sum_bound(s, dtype), "S")


def rows8(rows, cols, dtype, seed=0, pad=0, offset=0):
    g = _gen(seed)
    X = rows_of(g, rows, cols, dtype, pad, offset)
    (Q, whole), scale = eight_out(rows, cols, pad, offset), f32(rows)
    dg.quantize_rows_e4m3(X, Q, scale)
    assert eight_padding_intact(Q, whole, pad, offset)
    rr.assert_eight(Q, scale, X.double(), value=0.0)


def backward(rows, cols, dtype, affine=True, ds=True, in_place=False, seed=0, pad=0, offset=0, want=("dX", "dgamma")):
    g = _gen(seed)
    S, dY = rows_of(g, rows, cols, dtype, pad, offset), rows_of(g, rows, cols, dtype, pad, offset)
    dS = rows_of(g, rows, cols, dtype, pad, offset) if ds else None
    gamma = vector_of(g, cols, dtype) if affine else None
    rstd = (S.double().square().mean(1) + 1e-5).rsqrt().float()
    expected = rr.rms_grad(S, gamma, rstd, dY, dS)
    out = {"dX": dS if in_place else _out(rows, cols, dtype, pad, offset), "dgamma": f32(cols)}
    dg.rmsnorm_bwd(S, gamma, rstd, dY, dsum=dS, **{k: v for k, v in out.items() if k in want})
    for name, (v, bound) in expected.items():
        if name not in want:
            assert in_place or bool(torch.isnan(out[name]).all())
            continue
        if name == "dX":
            assert _padding_intact(out[name])
        ref.assert_within(out[name], v, bound, name)


SIZES = [(1, 1), (3, 1), (1, 2), (5, 7), (9, 31), (8, 32), (17, 33), (7, 100), (1, 256), (33, 257), (20, 512), (12, 1000), (3, 1025),
         (1, 4096), (300, 1537), (10, 4096), (5, 5001), (4, 8192), (2, 8200), (3, 16384), (2, 16391), (1, 40000)]
MANY = [(4097, 64), (3001, 264), (2500, 1000), (1000, 4096), (700, 9000)]   # more rows than blocks, in every shape of a row


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", SIZES + MANY)
def test_forward(size, dtype):
    forward(*size, dtype, seed=sum(size))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", SIZES + MANY)
def test_forward_to_8_bits(size, dtype):
    forward8(*size, dtype, seed=sum(size))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", SIZES + MANY)
def test_rows_to_8_bits(size, dtype):
    rows8(*size, dtype, seed=sum(size))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", SIZES + MANY)
def test_backward(size, dtype):
    backward(*size, dtype, seed=sum(size))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pad,offset", [(8, 0), (3, 0), (0, 1), (5, 3)])
@pytest.mark.parametrize("size", [(9, 100), (40, 1000), (600, 1000), (6, 5000), (3, 12000), (2, 20000)])
def test_strides_and_alignment(size, pad, offset, dtype):
    forward(*size, dtype, seed=pad, pad=pad, offset=offset)
    forward8(*size, dtype, seed=pad, pad=pad, offset=offset)
    rows8(*size, dtype, seed=pad, pad=pad, offset=offset)
    backward(*size, dtype, seed=pad, pad=pad, offset=offset)


@pytest.mark.parametrize("qpad,qoffset", [(0, 1), (1, 0), (4, 4), (8, 8), (0, 4)])
@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
@pytest.mark.parametrize("size", [(9, 96), (40, 1000), (2, 20000)])
def test_8_bits_at_any_address(size, dtype, qpad, qoffset):
    forward8(*size, dtype, qpad=qpad, qoffset=qoffset)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", [(5, 300), (600, 700), (6, 4096), (2, 20000)])
def test_optional_parts(size, dtype):
    forward(*size, dtype, res=False, keep=False)
    forward(*size, dtype, res=False, keep=True, affine=False)
    forward(*size, dtype, affine=False, stats=False, keep=False)
    forward8(*size, dtype, res=False, keep=False, affine=False)
    backward(*size, dtype, affine=False, ds=False)
    backward(*size, dtype, ds=False)
    backward(*size, dtype, want=("dX",))
    backward(*size, dtype, want=("dgamma",))


@pytest.mark.parametrize("pad", [0, 3])
@pytest.mark.parametrize("size", [(5, 300), (900, 700), (700, 4096), (7, 12000), (3, 20000)])
def test_outputs_in_the_place_of_inputs(size, pad):
    for dtype in (torch.bfloat16, torch.float32):
        for place in ("X", "R"):
            forward(*size, dtype, in_place=place, pad=pad)
            forward8(*size, dtype, in_place=place, pad=pad)
        forward(*size, dtype, res=False, in_place="X", pad=pad)
        backward(*size, dtype, in_place=True, pad=pad)


SHAPES = [(3, 40), (700, 200), (3, 600), (900, 1000), (4, 4096), (2, 9001), (2, 20000)]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dtype,size", [(torch.float32, 1e30), (torch.float32, 3e38), (torch.bfloat16, 1e25), (torch.float32, 1e-30), (torch.float32, 2e-43),
                                        (torch.bfloat16, 1e-35), (torch.float32, 2.0 ** 61), (torch.float32, 2.0 ** 64), (torch.float32, 2.0 ** -46)])
def test_rows_whose_squares_leave_the_range(shape, dtype, size):
    """Values whose squares overflow or vanish in binary32: with an eps that does not matter beside them, y is what it is for
    rows of ordinary size."""
    rows, cols = shape
    g = _gen(cols)
    X = (torch.rand(rows, cols, device="cuda", generator=g).double() * 2 - 1) * size
    X[:, 0] = size
    X = X.to(dtype)
    gamma = vector_of(g, cols, dtype)
    s, y, rstd = rr.rms(X, None, gamma, 0.0)
    Y, r = torch.empty_like(X), f32(rows)
    dg.rmsnorm_fwd(X, gamma, Y, eps=0.0, rstd=r)
    ref.assert_within(Y, y, rr.value_bound(y, dtype), "Y")
    inside = rstd < 3e38
    # rstd itself is subnormal from rows of 2^126 up: half a step of 2^-149
    ref.assert_within(r[inside], rstd[inside], rr.VALUE * rstd[inside] + 2.0 ** -149, "rstd")
    (Q, _), scale = eight_out(rows, cols), f32(rows)
    dg.rmsnorm_fwd_e4m3(X, gamma, Q, scale, eps=0.0)
    rr.assert_eight(Q, scale, y)


@pytest.mark.parametrize("shape", SHAPES)
def test_small_rows_under_an_eps(shape):
    """eps decides where rows are small: also where both are tiny."""
    for size, eps in ((1e-6, 1e-5), (1e-25, 1e-5), (1e-30, 1e-30), (1e-25, 1e-38), (1e-30, 1e-38)):
        X = torch.randn(*shape, device="cuda", generator=_gen(1)).double().mul(size).float()
        _, y, rstd = rr.rms(X, None, None, float(torch.tensor(eps, dtype=torch.float32)))
        Y, r = torch.empty_like(X), f32(shape[0])
        dg.rmsnorm_fwd(X, None, Y, eps=eps, rstd=r)
        ref.assert_within(Y, y, rr.value_bound(y, torch.float32), "Y")
        ref.assert_within(r, rstd, rr.VALUE * rstd, "rstd")


@pytest.mark.parametrize("shape", SHAPES)
def test_zero_rows(shape):
    X = torch.randn(*shape, device="cuda", generator=_gen(1)).bfloat16()
    X[1] = 0
    Y, r = torch.empty_like(X), f32(shape[0])
    (Q, _), scale = eight_out(*shape), f32(shape[0])
    dg.rmsnorm_fwd(X, None, Y, rstd=r)
    assert bool((Y[1] == 0).all()) and abs(float(r[1]) - 1e-5 ** -0.5) < 1e-3
    dg.rmsnorm_fwd_e4m3(X, None, Q, scale)
    least = float(torch.tensor(2.0 ** -100, dtype=torch.float32) / 448)
    assert bool((Q[1].float() == 0).all()) and float(scale[1]) == least
    dg.quantize_rows_e4m3(X, Q, scale)
    assert bool((Q[1].float() == 0).all()) and float(scale[1]) == least
    # without an eps a zero row has no norm: NaN there, and nowhere else
    dg.rmsnorm_fwd(X, None, Y, eps=0.0, rstd=r)
    assert bool(torch.isnan(Y[1]).all()) and bool(torch.isfinite(Y[0]).all()) and bool(torch.isinf(r[1]))


@pytest.mark.parametrize("shape", SHAPES)
def test_nan_and_infinity_stay_in_their_row(shape):
    g = _gen(5)
    rows, cols = shape
    for value in (NAN, INF, -INF):
        X, R = rows_of(g, rows, cols, torch.bfloat16), rows_of(g, rows, cols, torch.bfloat16)
        X[1, cols - 1] = value
        Y, S, r = torch.empty_like(X), torch.empty_like(X), f32(rows)
        dg.rmsnorm_fwd(X, None, Y, residual=R, sum=S, rstd=r)
        s = X.float() + R.float()
        want = s * torch.rsqrt((s * s).mean(1, keepdim=True) + 1e-5)
        assert torch.equal(torch.isnan(Y), torch.isnan(want)) and bool(torch.isfinite(Y[0]).all())
        if value == value:
            assert bool((Y[1, :cols - 1] == 0).all()) and float(r[1]) == 0.0
        (Q, _), scale = eight_out(rows, cols), f32(rows)
        dg.rmsnorm_fwd_e4m3(X, None, Q, scale, residual=R)
        assert bool(torch.isnan(scale[1])) and bool(torch.isnan(Q[1].float()).all()) and bool(torch.isfinite(Q[0].float()).all())
        dg.quantize_rows_e4m3(X, Q, scale)
        assert not bool(torch.isfinite(scale[1])) and bool(torch.isnan(Q[1, cols - 1].float())) and bool(torch.isfinite(Q[0].float()).all())
        # backward: the gradient of the row alone, and of its column's weight
        dX, dga = torch.empty_like(X), f32(cols)
        rstd = torch.ones(rows, device="cuda")
        dg.rmsnorm_bwd(X, None, rstd, R, dX=dX, dgamma=dga)
        want = rr.rms_grad(X, None, rstd, R, None)["dX"][0]      # an infinite sum: infinities in the whole row, NaN at the place itself
        assert bool(torch.isfinite(dX[0]).all()) and torch.equal(torch.isnan(dX), torch.isnan(want)) and torch.equal(torch.isinf(dX), torch.isinf(want))
        assert not bool(torch.isfinite(dga[cols - 1])) and bool(torch.isfinite(dga[:cols - 1]).all())


@pytest.mark.parametrize("cols", [33, 1001, 4100, 9001, 17000])
@pytest.mark.parametrize("dtype", TYPES)
def test_an_infinite_statistic_stays_in_its_row(cols, dtype):
    """rstd of a zero row without an eps is infinite: what lies beyond the row's end must not make it NaN elsewhere."""
    S = torch.randn(5, cols, device="cuda", generator=_gen(1)).to(dtype)
    dY = torch.randn(5, cols, device="cuda", generator=_gen(2)).to(dtype)
    rstd = torch.ones(5, device="cuda")
    rstd[2] = INF
    S[2], dY[2] = 1, 0
    dX = torch.empty_like(S)
    dg.rmsnorm_bwd(S, None, rstd, dY, dX=dX)
    assert bool(torch.isfinite(dX[[0, 1, 3, 4]]).all()) and bool(torch.isnan(dX[2]).all())


def test_ties_and_ends_of_8_bits():
    """Every e4m3 value, the points half-way between two of them and their neighbours: nearest, ties to even, in a row whose scale is 1."""
    every = torch.arange(127, dtype=torch.uint8, device="cuda").view(rr.E4M3).float()          # 0 .. 448
    mid = (every[1:] + every[:-1]) / 2
    row = torch.cat([every, mid, torch.nextafter(mid, mid * 2), torch.nextafter(mid, mid * 0)])
    row = torch.cat([row, -row])[None].contiguous()
    (Q, _), scale = eight_out(*row.shape), f32(1)
    dg.quantize_rows_e4m3(row, Q, scale)
    assert float(scale) == 1.0
    v = row.double()
    step = 2 * rr.half_step(v)
    assert torch.equal(Q.double(), torch.round(v / step) * step)


def test_same_bits_every_time():
    g = _gen(6)
    S, dY = rows_of(g, 3000, 1000, torch.bfloat16), rows_of(g, 3000, 1000, torch.bfloat16)
    rstd = (S.float().square().mean(1) + 1e-5).rsqrt()
    runs = []
    for _ in range(5):
        dX, a = torch.empty_like(S), f32(1000)
        dg.rmsnorm_bwd(S, None, rstd, dY, dsum=dY.clone(), dX=dX, dgamma=a)
        runs.append((dX, a))
    for r in runs[1:]:
        assert all(torch.equal(x, y) for x, y in zip(r, runs[0]))


@pytest.mark.parametrize("cols", [90, 1111, 9000, 17001])
def test_gradient_agrees_with_differences(cols):
    g = _gen(7)
    X, R, dY, dS = (rows_of(g, 6, cols, torch.float32) for _ in range(4))
    gamma = vector_of(g, cols, torch.float32)
    Y, S, r = torch.empty_like(X), torch.empty_like(X), f32(6)
    dg.rmsnorm_fwd(X, gamma, Y, residual=R, sum=S, rstd=r)
    dX, dga = torch.empty_like(X), f32(cols)
    dg.rmsnorm_bwd(S, gamma, r, dY, dsum=dS, dX=dX, dgamma=dga)
    E = [torch.randn(*s, device="cuda", generator=g).double() for s in ((6, cols), (6, cols), (cols,))]

    def f(t):
        s, y, _ = rr.rms(X.double() + t * E[0], R.double() + t * E[1], gamma.double() + t * E[2], 1e-5)
        return float((dY.double() * y).sum() + (dS.double() * s).sum())

    h = 1e-5
    slope = (f(h) - f(-h)) / (2 * h)
    parts = [dX.double() * E[0], dX.double() * E[1], dga.double() * E[2]]
    # every gradient is known to 2^-18 or so of its size in binary32; the differences to h^2
    assert abs(sum(float(p.sum()) for p in parts) - slope) <= 2.0 ** -17 * sum(float(p.abs().sum()) for p in parts) + 1e-5


def test_empty_and_refusals():
    bf = torch.bfloat16
    e = lambda *s, t=bf: torch.zeros(*s, dtype=t, device="cuda")   # noqa: E731
    dg.rmsnorm_fwd(e(0, 8), None, e(0, 8))
    dg.rmsnorm_fwd(e(4, 0), None, e(4, 0))
    dg.quantize_rows_e4m3(e(0, 8), e(0, 8, t=rr.E4M3), e(0, t=torch.float32))
    a = f32(8)
    dg.rmsnorm_bwd(e(0, 8), None, e(0, t=torch.float32), e(0, 8), dgamma=a)
    assert bool((a == 0).all())
    X, Y = e(4, 8), e(4, 8)
    with pytest.raises(dg.DgemmError):
        dg.rmsnorm_fwd(X, None, X)
    with pytest.raises(dg.DgemmError):
        dg.rmsnorm_fwd(X, None, Y, eps=-1.0)
    with pytest.raises(dg.DgemmError):
        dg.rmsnorm_bwd(X, None, None, Y, dX=e(4, 8))
    with pytest.raises(TypeError):
        dg.rmsnorm_fwd(X, torch.ones(8, device="cuda"), Y)
    with pytest.raises(TypeError):
        dg.rmsnorm_fwd(X, None, Y, residual=X.float())
    with pytest.raises(ValueError):
        dg.rmsnorm_fwd(X, None, Y, residual=e(4, 9))
    with pytest.raises(TypeError):
        dg.quantize_rows_e4m3(X, Y, f32(4))
    with pytest.raises(ValueError):
        dg.rmsnorm_fwd_e4m3(X, None, e(4, 8, t=rr.E4M3), f32(3))
    with pytest.raises(ValueError):
        dg.rmsnorm_fwd(X.t(), None, e(8, 4))     # columns are not contiguous
