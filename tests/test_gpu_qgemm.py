"""The products of 8-bit operands and the gated projections against plain 64-bit forms (bounds: ``rows_reference``); on small-integer
data with scales that are powers of two all sums are exact and the outputs must be the rounded exact values bit for bit. Needs a B200."""
import pytest
import torch

import hgemm_reference as ref
import paper_2003_00532_b200 as dg
import rows_reference as rr
from test_gpu_hgemm import _draw, _gen, _ok, _out, _padding_intact

pytestmark = pytest.mark.gpu

TYPES = [torch.bfloat16, torch.float16]
NAN = float("nan")


def eight(g, rows, cols, integer=False, pad=0, offset=0):
    """An 8-bit matrix in a buffer of NaN bytes."""
    ld = cols + pad
    whole = torch.full((rows * ld + offset + 16,), 0x7f, dtype=torch.uint8, device="cuda").view(rr.E4M3)
    view = whole[offset:offset + rows * ld].view(rows, ld)[:, :cols]
    x = torch.randint(-4, 5, (rows, cols), device="cuda", generator=g).float() if integer else torch.randn(rows, cols, device="cuda", generator=g) * 100
    view.copy_(x.clamp(-448, 448).to(rr.E4M3))
    return view


def scales(g, n, integer=False, mid=1.0):
    if integer:
        return torch.exp2(torch.randint(-1, 2, (n,), device="cuda", generator=g).float())
    return (torch.rand(n, device="cuda", generator=g) + 0.5) * mid


def _linear(M, N, K, dtype, act=ref.NONE, bias=True, res=True, save=True, sa=True, sb=True, integer=False, pad=0, offset=0, qpad=None, in_place=False, seed=0):
    g = _gen(seed)
    qpad = pad if qpad is None else qpad
    A, B = eight(g, M, K, integer, qpad, offset), eight(g, N, K, integer, qpad, offset)
    a = scales(g, M, integer, 0.01) if sa else None
    b = scales(g, N, integer, 0.01 * K ** -0.5) if sb else None
    c = _draw(g, 1, N, dtype, 0.5, integer)[0] if bias else None
    R = _draw(g, M, N, dtype, 1.0, integer, pad, offset) if res else None
    D = R if in_place else _out(M, N, dtype, pad, offset)
    Z = _out(M, N, dtype, pad, offset) if save else None
    want, bound, z, zbound = rr.linear8(A, B, a, b, c, act, R, dtype)
    dg.qgemm_epilogue(A, B, D, a_scale=a, b_scale=b, bias=c, act=act, residual=R, preact=Z)
    _ok()
    assert _padding_intact(D) and (Z is None or _padding_intact(Z)), "padding was written"
    if integer and act in (ref.NONE, ref.RELU):
        assert torch.equal(D.contiguous(), want.to(dtype)), "integer data: not the rounded exact value"
    ref.assert_within(D, want, bound, "D")
    if save:
        ref.assert_within(Z, z, zbound, "Z")


def _gated(M, F, K, dtype, act=ref.SILU, save=True, scaled=True, integer=False, pad=0, offset=0, qpad=None, seed=0):
    g = _gen(seed)
    qpad = pad if qpad is None else qpad
    X, Wg, Wu = eight(g, M, K, integer, qpad, offset), eight(g, F, K, integer, qpad, offset), eight(g, F, K, integer, qpad, offset)
    sx, sg, su = (scales(g, n, integer, m) if scaled else None for n, m in ((M, 0.01), (F, 0.01 * K ** -0.5), (F, 0.01 * K ** -0.5)))
    out = {k: _out(M, F, dtype, pad, offset) for k in ("H", "G", "U")}
    want = rr.gated8(X, Wg, Wu, sx, sg, su, act, dtype)
    dg.qgemm_gated(X, Wg, Wu, out["H"], x_scale=sx, g_scale=sg, u_scale=su, act=act, **({"gate": out["G"], "up": out["U"]} if save else {}))
    _ok()
    for name, (v, bound) in want.items():
        if name != "H" and not save:
            continue
        assert _padding_intact(out[name])
        if integer and act in (ref.NONE, ref.RELU):
            assert torch.equal(out[name].contiguous(), v.to(dtype)), name   # (infinite where a product leaves binary16)
        else:
            ref.assert_within(out[name], v, bound, name)


SHAPES = [(1, 1, 1), (1, 64, 64), (2, 7, 5), (3, 130, 65), (16, 128, 128), (17, 129, 127), (33, 500, 200), (64, 256, 128), (65, 100, 1000),
          (128, 128, 128), (129, 257, 129), (256, 256, 256), (300, 260, 200), (1000, 1537, 777), (515, 31, 4099), (37, 4000, 515)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_linear_exact_on_integers(shape, dtype):
    _linear(*shape, dtype, integer=True, seed=sum(shape))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_linear(shape, dtype):
    _linear(*shape, dtype, act=ref.GELU_TANH, seed=sum(shape))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_gated(shape, dtype):
    _gated(*shape, dtype, ref.NONE, integer=True, seed=sum(shape))
    _gated(*shape, dtype, ref.SILU, seed=sum(shape))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pad,offset", [(0, 0), (16, 0), (3, 0), (0, 1), (8, 8)])
@pytest.mark.parametrize("shape", [(1, 4096, 333), (2, 3001, 208), (3, 3333, 77), (4, 3500, 700), (4, 5, 9001), (1, 70, 20000), (3, 1, 8), (8, 1000, 4096)])
def test_few_rows(shape, pad, offset, dtype):
    _linear(*shape, dtype, integer=True, seed=sum(shape), pad=pad, offset=offset)
    _linear(*shape, dtype, act=ref.SILU, res=False, save=False, seed=1, pad=pad, offset=offset)
    _gated(*shape, dtype, ref.RELU, integer=True, seed=sum(shape), pad=pad, offset=offset)
    _gated(*shape, dtype, ref.SILU, save=False, seed=2, pad=pad, offset=offset)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("act", ref.ACTS)
@pytest.mark.parametrize("shape", [(1, 300, 500), (130, 200, 300), (600, 520, 96)])
def test_activations(shape, act, dtype):
    _linear(*shape, dtype, act=act, seed=act)
    _gated(*shape, dtype, act, seed=act)


@pytest.mark.parametrize("bias,res,save,sa,sb", [(False, False, False, True, True), (True, False, False, False, True), (False, True, False, True, False),
                                                 (False, False, True, False, False), (True, True, True, False, False)])
@pytest.mark.parametrize("shape", [(5, 200, 3000), (700, 300, 200)])
def test_optional_parts(shape, bias, res, save, sa, sb):
    _linear(*shape, torch.bfloat16, ref.NONE, bias, res, save, sa, sb, seed=7)
    _gated(*shape, torch.bfloat16, ref.NONE, save=save, scaled=sa, integer=True, seed=7)


@pytest.mark.parametrize("pad,offset,qpad", [(8, 0, 16), (3, 0, 3), (0, 1, 0), (5, 4, 1), (8, 8, 8), (8, 3, 16), (0, 0, 2)])
@pytest.mark.parametrize("shape", [(9, 200, 136), (260, 264, 336), (70, 100, 19), (70, 100, 16)])
def test_strides_and_alignment(shape, pad, offset, qpad):
    _linear(*shape, torch.float16, integer=True, seed=pad + offset, pad=pad, offset=offset, qpad=qpad)
    _gated(*shape, torch.bfloat16, ref.NONE, integer=True, seed=pad, pad=pad, offset=offset, qpad=qpad)


@pytest.mark.parametrize("shape", [(1, 512, 4096), (40, 300, 5000), (300, 300, 6000)])
def test_residual_in_place(shape):
    """R may be D; also where the tile's k-blocks are cut into parts."""
    _linear(*shape, torch.bfloat16, ref.SILU, True, True, False, seed=5, in_place=True, pad=8)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", [(1, 4096, 4096), (64, 1024, 8192), (200, 2048, 4096), (2088, 2088, 2088), (4097, 31, 4099), (1024, 4096, 512)])
def test_large(shape, dtype):
    _linear(*shape, dtype, ref.GELU_TANH, True, False, True, seed=11)


def test_wide_tiles():
    """Long contractions over several rounds run on 512 x 256 tiles."""
    M, N, K = 3700, 7900, 12600
    assert dg.hgemm_plan(M, N, (K + 1) // 2)["tile_cols"] == 512
    _linear(M, N, K, torch.bfloat16, integer=True, seed=1)
    assert dg.hgemm_plan(M, 4000, (K + 1) // 2, gated=True)["tile_cols"] == 256
    _gated(M, 4000, K, torch.float16, seed=2)


def test_every_8_bit_value():
    """All 256 codes, NaN among them, against ones: each row's product is its value."""
    codes = torch.arange(256, dtype=torch.uint8, device="cuda").view(rr.E4M3)
    A = torch.zeros(256, 160, dtype=rr.E4M3, device="cuda")
    A[:, 77] = codes
    B = torch.ones(40, 160, device="cuda").to(rr.E4M3)
    D = torch.empty(256, 40, dtype=torch.bfloat16, device="cuda")
    for x, w, out in ((A, B, D), (B, A, torch.empty(40, 256, dtype=torch.bfloat16, device="cuda"))):
        dg.qgemm_epilogue(x, w, out)
        want = codes.float().bfloat16()
        got = out[:, 0] if out is D else out[0]
        assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got[~torch.isnan(want)], want[~torch.isnan(want)])
    _ok()


def test_nan_and_infinite_scales_stay_in_their_row_and_column():
    g = _gen(4)
    A, B = eight(g, 50, 300), eight(g, 90, 300)
    a, b = scales(g, 50), scales(g, 90)
    a[3], a[7], b[11] = NAN, float("inf"), NAN
    D = torch.empty(50, 90, dtype=torch.bfloat16, device="cuda")
    dg.qgemm_epilogue(A, B, D, a_scale=a, b_scale=b)
    bad = torch.zeros(50, 90, dtype=torch.bool, device="cuda")
    bad[3], bad[7], bad[:, 11] = True, True, True
    assert torch.equal(~torch.isfinite(D), bad)


def test_extreme_scales():
    """The largest and smallest scales that rows in 8 bits get: their product may leave binary32's range where the result does not."""
    g = _gen(4)
    A, B = eight(g, 20, 64, integer=True), eight(g, 30, 64, integer=True)
    a, b = torch.full((20,), 2.0 ** -109, device="cuda"), torch.full((30,), 2.0 ** 100, device="cuda")
    D = torch.empty(20, 30, dtype=torch.bfloat16, device="cuda")
    dg.qgemm_epilogue(A, B, D, a_scale=a, b_scale=b)
    assert torch.equal(D.double(), (A.double() @ B.double().t() * 2.0 ** -9).bfloat16().double())


def test_large_sums_keep_their_bits():
    """A sum of products that cancel: 448 x 448 and small values beside them are added in binary32."""
    K = 512
    A, B = torch.zeros(4, K, device="cuda"), torch.zeros(8, K, device="cuda")
    A[:, 0], A[:, 200], A[:, 400] = 448, -448, 0.015625
    B[:, 0], B[:, 200], B[:, 400] = 448, 448, 0.015625 * 64
    D = torch.empty(4, 8, dtype=torch.float16, device="cuda")
    dg.qgemm_epilogue(A.to(rr.E4M3), B.to(rr.E4M3), D)
    assert bool((D == 0.015625).all())


def test_empty():
    bf = torch.bfloat16
    q = lambda *s: torch.zeros(*s, device="cuda").to(rr.E4M3)   # noqa: E731
    bias = torch.randn(6, device="cuda").to(bf)
    R, D = torch.randn(4, 6, device="cuda").to(bf), torch.empty(4, 6, dtype=bf, device="cuda")
    dg.qgemm_epilogue(q(4, 0), q(6, 0), D, bias=bias, act=dg.HGEMM_ACT_RELU, residual=R)
    assert torch.equal(D, (bias.float().clamp_min(0) + R.float()).to(bf))
    H, G, U = (torch.full((4, 6), NAN, dtype=bf, device="cuda") for _ in range(3))
    dg.qgemm_gated(q(4, 0), q(6, 0), q(6, 0), H, gate=G, up=U)
    assert all(bool((x == 0).all()) for x in (H, G, U))
    dg.qgemm_epilogue(q(0, 8), q(6, 8), torch.empty(0, 6, dtype=bf, device="cuda"))
    dg.qgemm_epilogue(q(4, 8), q(0, 8), torch.empty(4, 0, dtype=bf, device="cuda"))


def test_refusals():
    bf = torch.bfloat16
    q = lambda *s: torch.zeros(*s, device="cuda").to(rr.E4M3)   # noqa: E731
    D = torch.empty(4, 6, dtype=bf, device="cuda")
    with pytest.raises(TypeError):
        dg.qgemm_epilogue(torch.zeros(4, 8, dtype=bf, device="cuda"), q(6, 8), D)
    with pytest.raises(ValueError):
        dg.qgemm_epilogue(q(4, 8), q(6, 9), D)
    with pytest.raises(ValueError):
        dg.qgemm_epilogue(q(8, 4).t(), q(6, 8), D)
    with pytest.raises(TypeError):
        dg.qgemm_epilogue(q(4, 8), q(6, 8), D, a_scale=torch.ones(4, device="cuda", dtype=bf))
    with pytest.raises(ValueError):
        dg.qgemm_epilogue(q(4, 8), q(6, 8), D, b_scale=torch.ones(4, device="cuda"))
    with pytest.raises(dg.DgemmError):
        dg.qgemm_epilogue(q(4, 8), q(6, 8), torch.empty(4, 6, device="cuda"))
    with pytest.raises(dg.DgemmError):
        dg.qgemm_gated(q(4, 8), q(6, 8), q(6, 8), D, gate=torch.empty_like(D))
