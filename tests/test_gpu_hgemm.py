"""The 16-bit products with an epilogue and the gated projections, forward and backward, against plain
64-bit forms. Needs a B200. The bounds are derived in ``hgemm_reference``; on small-integer data all
sums are exact and the outputs must be the rounded exact values bit for bit."""
import pytest
import torch

import hgemm_reference as ref
import paper_2003_00532_b200 as dg

pytestmark = pytest.mark.gpu

TYPES = [torch.bfloat16, torch.float16]


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _place(x, pad=0, offset=0):
    """x in a wider NaN-filled buffer whose first element is `offset` elements off an aligned address."""
    rows, cols = x.shape
    ld = cols + pad
    whole = torch.full((rows * ld + offset + 8,), float("nan"), dtype=x.dtype, device="cuda")
    view = whole[offset:offset + rows * ld].view(rows, ld)
    view[:, :cols] = x
    return view[:, :cols]


def _draw(g, rows, cols, dtype, scale=1.0, integer=False, pad=0, offset=0):
    if integer:
        x = torch.randint(-4, 5, (rows, cols), device="cuda", generator=g).to(dtype)
    else:
        x = (torch.randn(rows, cols, device="cuda", generator=g) * scale).to(dtype)
    return _place(x, pad, offset)


def _out(rows, cols, dtype, pad=0, offset=0):
    return _place(torch.full((rows, cols), float("nan"), dtype=dtype, device="cuda"), pad, offset)


def _padding_intact(view):
    rows, cols = view.shape
    ld = view.stride(0)
    if rows < 2 or ld == cols:
        return True
    whole = view.as_strided((rows - 1, ld), (ld, 1))
    return bool(torch.isnan(whole[:, cols:]).all())


def _ok():
    assert dg.hgemm_last_device_status() == dg.DGEMM_OK


def _linear_case(M, N, K, dtype, transa, transb, act, bias, res, save, seed=0, integer=False, pad=0, offset=0, in_place=False):
    g = _gen(seed)
    scale = K ** -0.5
    A = _draw(g, *((K, M) if transa else (M, K)), dtype, 1.0, integer, pad, offset)
    B = _draw(g, *((N, K) if transb else (K, N)), dtype, scale, integer, pad, offset)
    b = _draw(g, 1, N, dtype, 0.5, integer)[0] if bias else None
    R = _draw(g, M, N, dtype, 1.0, integer, pad, offset) if res else None
    D = R if in_place else _out(M, N, dtype, pad, offset)
    Z = _out(M, N, dtype, pad, offset) if save else None
    want, bound, z, zbound = ref.linear(A, B, b, act, R, transa, transb)
    dg.hgemm_epilogue(A, B, D, bias=b, act=act, residual=R, preact=Z, transa=transa, transb=transb)
    _ok()
    assert _padding_intact(D) and (Z is None or _padding_intact(Z)), "padding was written"
    if integer and act in (ref.NONE, ref.RELU):
        assert torch.equal(D.contiguous(), want.to(dtype)), "integer data: not the rounded exact value"
    ref.assert_within(D, want, bound, "D")
    if save:
        ref.assert_within(Z, z, zbound, "Z")


SHAPES = [(1, 1, 1), (1, 64, 64), (2, 7, 5), (3, 130, 65), (16, 128, 64), (17, 129, 63), (33, 500, 200), (64, 256, 128), (65, 100, 1000),
          (128, 128, 128), (129, 257, 65), (256, 256, 256), (300, 260, 200), (1000, 1537, 777), (515, 31, 4099), (37, 4000, 515)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("transa", [False, True])
@pytest.mark.parametrize("transb", [False, True])
@pytest.mark.parametrize("shape", SHAPES)
def test_linear_exact_on_integers(shape, transa, transb, dtype):
    _linear_case(*shape, dtype, transa, transb, ref.NONE, True, True, True, seed=sum(shape), integer=True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("transa,transb", [(False, False), (False, True), (True, False), (True, True)])
@pytest.mark.parametrize("pad,offset", [(0, 0), (8, 0), (3, 0), (0, 1)])
@pytest.mark.parametrize("shape", [(1, 4096, 333), (2, 3001, 200), (3, 3333, 77), (4, 3500, 700), (4, 5, 9001), (1, 70, 20000), (3, 1, 8)])
def test_linear_of_few_rows(shape, pad, offset, transa, transb, dtype):
    """One to four rows; one and two have a kernel of their own for aligned weights stored N x K."""
    _linear_case(*shape, dtype, transa, transb, ref.NONE, True, True, True, seed=sum(shape), integer=True, pad=pad, offset=offset)
    _linear_case(*shape, dtype, transa, transb, ref.SILU, True, False, False, seed=1, pad=pad, offset=offset)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("act", ref.ACTS)
@pytest.mark.parametrize("shape", [(1, 300, 500), (130, 200, 300), (600, 520, 96)])
def test_linear_activations(shape, act, dtype):
    _linear_case(*shape, dtype, False, True, act, True, True, True, seed=act)


@pytest.mark.parametrize("bias,res,save", [(False, False, False), (True, False, False), (False, True, False), (False, False, True)])
@pytest.mark.parametrize("shape", [(5, 200, 3000), (700, 300, 200)])
def test_linear_optional_parts(shape, bias, res, save):
    _linear_case(*shape, torch.bfloat16, False, False, ref.GELU, bias, res, save, seed=7)


@pytest.mark.parametrize("transa,transb", [(False, False), (False, True), (True, False), (True, True)])
@pytest.mark.parametrize("pad,offset", [(8, 0), (3, 0), (0, 1), (5, 4), (8, 8)])
@pytest.mark.parametrize("shape", [(9, 200, 136), (260, 264, 328)])
def test_linear_strides_and_alignment(shape, pad, offset, transa, transb):
    _linear_case(*shape, torch.float16, transa, transb, ref.NONE, True, True, True, seed=pad + offset, integer=True, pad=pad, offset=offset)


@pytest.mark.parametrize("shape", [(1, 512, 4096), (40, 300, 5000), (300, 300, 3000)])
def test_linear_residual_in_place(shape):
    """R may be D; also where the tile's k-blocks are cut into parts."""
    _linear_case(*shape, torch.bfloat16, False, True, ref.SILU, True, True, False, seed=5, in_place=True, pad=8)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", [(1, 4096, 4096), (64, 1024, 8192), (200, 2048, 4096), (2088, 2088, 2088), (4097, 31, 4099), (1024, 4096, 512)])
def test_linear_large(shape, dtype):
    _linear_case(*shape, dtype, False, True, ref.GELU_TANH, True, False, True, seed=11)


WIDE = (3700, 7900, 6300)  # long contraction, several rounds of 512 x 256 tiles, ragged in every direction


@pytest.mark.parametrize("transa,transb", [(False, True), (True, False)])
def test_linear_wide_tiles(transa, transb):
    assert dg.hgemm_plan(*WIDE)["tile_cols"] == 512
    _linear_case(*WIDE, torch.bfloat16, transa, transb, ref.NONE, True, True, True, seed=1, integer=True)


def test_gated_wide_tiles():
    M, F, K = 3700, 4000, 6300
    assert dg.hgemm_plan(M, F, K, gated=True)["tile_cols"] == 256
    _gated_case(M, F, K, torch.float16, True, ref.SILU, True, seed=2)
    _gated_case(M, F, K, torch.bfloat16, False, ref.GELU_TANH, False, seed=3)


def test_gradients_wide_tiles():
    _gated_grad_case(6200, 8100, 2000, torch.bfloat16, False, ref.SILU, seed=4)
    _linear_grad_case(7000, 6700, 7100, torch.float16, False, True, ref.NONE, seed=5)


def test_repeated_calls_give_the_same_bits():
    """Cut tiles are added in a fixed order, whichever part finishes last."""
    g = _gen(3)
    for M, N, K in ((1, 1024, 8192), (300, 700, 6000)):
        A, B = _draw(g, M, K, torch.bfloat16), _draw(g, N, K, torch.bfloat16, K ** -0.5)
        assert dg.hgemm_plan(M, N, K)["span"] > 0
        first = None
        for _ in range(20):
            D = _out(M, N, torch.bfloat16)
            dg.hgemm_epilogue(A, B, D, transb=True)
            first = D if first is None else first
            assert torch.equal(D, first)
    _ok()


def test_infinities_and_nan_stay_in_their_rows_and_columns():
    g = _gen(4)
    M, N, K = 150, 140, 70
    A, B = _draw(g, M, K, torch.float16), _draw(g, N, K, torch.float16, 0.1)
    A[3, 5], A[77, 69], B[130, 0] = float("inf"), float("nan"), float("nan")
    D = _out(M, N, torch.float16)
    dg.hgemm_epilogue(A, B, D, act=dg.HGEMM_ACT_RELU, transb=True)
    bad = torch.zeros(M, N, dtype=torch.bool, device="cuda")
    bad[77], bad[:, 130] = True, True
    assert bool(torch.isnan(D[bad]).all())
    rest = ~bad
    rest[3] = False
    assert bool(torch.isfinite(D[rest]).all())
    row = D[3][torch.arange(N, device="cuda") != 130]
    assert bool(((row == float("inf")) | (row == 0)).all())


def test_empty_sums_and_empty_outputs():
    bf = torch.bfloat16
    b = torch.randn(70, device="cuda").to(bf)
    R = torch.randn(5, 70, device="cuda").to(bf)
    D, Z = _out(5, 70, bf), _out(5, 70, bf)
    A0, B0 = torch.zeros(5, 0, dtype=bf, device="cuda"), torch.zeros(0, 70, dtype=bf, device="cuda")
    dg.hgemm_epilogue(A0, B0, D, bias=b, act=dg.HGEMM_ACT_SILU, residual=R, preact=Z)
    want = ref.act(b.double(), ref.SILU)[None, :] + R.double()
    ref.assert_within(D, want, ref.rounded(want, 2.0 ** -19 * (b.double().abs() + R.double().abs()), bf), "D")
    assert torch.equal(Z, b[None, :].expand(5, 70))
    dg.hgemm_epilogue(torch.zeros(0, 8, dtype=bf, device="cuda"), torch.zeros(8, 70, dtype=bf, device="cuda"), torch.zeros(0, 70, dtype=bf, device="cuda"))
    # no rows: the weight's and the bias's gradients are zero; no columns: the input's
    dB, db = _out(8, 70, bf), torch.full((70,), float("nan"), device="cuda")
    dg.hgemm_epilogue_bwd(torch.zeros(0, 8, dtype=bf, device="cuda"), torch.zeros(8, 70, dtype=bf, device="cuda"),
                          torch.zeros(0, 70, dtype=bf, device="cuda"), dB=dB, dbias=db)
    assert bool((dB == 0).all()) and bool((db == 0).all())
    dA = _out(5, 8, bf)
    dg.hgemm_epilogue_bwd(torch.zeros(5, 8, dtype=bf, device="cuda"), torch.zeros(8, 0, dtype=bf, device="cuda"),
                          torch.zeros(5, 0, dtype=bf, device="cuda"), dA=dA)
    assert bool((dA == 0).all())
    H, G, U = _out(3, 9, bf), _out(3, 9, bf), _out(3, 9, bf)
    dg.hgemm_gated(torch.zeros(3, 0, dtype=bf, device="cuda"), torch.zeros(0, 9, dtype=bf, device="cuda"), torch.zeros(0, 9, dtype=bf, device="cuda"),
                   H, gate=G, up=U)
    assert bool((H == 0).all()) and bool((G == 0).all()) and bool((U == 0).all())
    _ok()


# ---- gradients of the product ----------------------------------------------------------------------

def _linear_grad_case(M, N, K, dtype, transa, transb, act, seed=0, integer=False, pad=0, offset=0, want=("dA", "dB", "dbias")):
    g = _gen(seed)
    A = _draw(g, *((K, M) if transa else (M, K)), dtype, 1.0, integer, pad, offset)
    B = _draw(g, *((N, K) if transb else (K, N)), dtype, K ** -0.5, integer, pad, offset)
    dD = _draw(g, M, N, dtype, 0.1, integer, pad, offset)
    Z = _draw(g, M, N, dtype, 1.5, integer, pad, offset) if act != ref.NONE else None
    out = {"dA": _out(*A.shape, dtype, pad, offset), "dB": _out(*B.shape, dtype, pad, offset), "dbias": torch.full((N,), float("nan"), device="cuda")}
    args = {k: v for k, v in out.items() if k in want}
    dg.hgemm_epilogue_bwd(A, B, dD, act=act, preact=Z, transa=transa, transb=transb, **args)
    _ok()
    for name, (v, bound) in ref.linear_grad(A, B, Z, act, dD, transa, transb).items():
        if name not in want:
            assert bool(torch.isnan(out[name]).all())
            continue
        assert out[name].dim() == 1 or _padding_intact(out[name])
        if integer and act in (ref.NONE, ref.RELU):
            assert torch.equal(out[name].contiguous(), v.to(out[name].dtype)), name
        ref.assert_within(out[name], v, bound, name)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("transa", [False, True])
@pytest.mark.parametrize("transb", [False, True])
@pytest.mark.parametrize("shape", [(1, 1, 1), (1, 200, 300), (5, 66, 129), (130, 257, 70), (300, 64, 500), (1000, 1537, 777)])
def test_linear_gradients_exact_on_integers(shape, transa, transb, dtype):
    _linear_grad_case(*shape, dtype, transa, transb, ref.RELU, seed=sum(shape), integer=True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("act", ref.ACTS)
@pytest.mark.parametrize("shape", [(3, 200, 100), (520, 264, 328)])
def test_linear_gradients_activations(shape, act, dtype):
    _linear_grad_case(*shape, dtype, False, True, act, seed=act)


@pytest.mark.parametrize("want", [("dA",), ("dB",), ("dbias",), ("dA", "dbias"), ("dA", "dB")])
@pytest.mark.parametrize("act", [ref.NONE, ref.SILU])
def test_linear_gradients_optional_outputs(want, act):
    _linear_grad_case(77, 200, 90, torch.bfloat16, False, False, act, seed=2, want=want)


@pytest.mark.parametrize("act", [ref.NONE, ref.RELU])
@pytest.mark.parametrize("pad,offset", [(8, 0), (3, 0), (0, 1), (5, 3)])
@pytest.mark.parametrize("transa,transb", [(False, False), (True, True)])
def test_linear_gradients_strides_and_alignment(transa, transb, pad, offset, act):
    _linear_grad_case(200, 136, 264, torch.float16, transa, transb, act, seed=9, integer=True, pad=pad, offset=offset)


def test_linear_gradients_large():
    _linear_grad_case(2088, 4096, 1024, torch.bfloat16, False, True, ref.GELU_TANH, seed=1)
    _linear_grad_case(4099, 96, 2048, torch.float16, False, False, ref.GELU, seed=1)


def test_linear_gradient_agrees_with_differences():
    """d/dt of sum(dD * D(A + t E, B, b)) by central differences of the 64-bit form, against the kernel's dA and dbias."""
    g = _gen(8)
    M, N, K, t = 40, 60, 50, torch.float16
    A, B, b = _draw(g, M, K, t), _draw(g, N, K, t, 0.2), _draw(g, 1, N, t, 0.5)[0]
    dD = _draw(g, M, N, t, 0.5)
    for act in (ref.GELU, ref.GELU_TANH, ref.SILU):
        D, Z = _out(M, N, t), _out(M, N, t)
        dg.hgemm_epilogue(A, B, D, bias=b, act=act, preact=Z, transb=True)
        dA, db = _out(M, K, t), torch.empty(N, device="cuda")
        dg.hgemm_epilogue_bwd(A, B, dD, act=act, preact=Z, dA=dA, dbias=db, transb=True)
        E, e = torch.randn(M, K, device="cuda", generator=g).double(), torch.randn(N, device="cuda", generator=g).double()

        def f(s):
            z = (A.double() + s * E) @ B.double().t() + b.double() + s * e
            return float((dD.double() * ref.act(z, act)).sum())

        h = 1e-4
        slope = (f(h) - f(-h)) / (2 * h)
        got = float((dA.double() * E).sum() + (db.double() * e).sum())
        # Z, dZ and dA are each rounded once (2^-11 of their size; |act''| <= 1.13 for Z): a sum of M K terms
        zr = ref.linear(A, B, b, act, None, False, True)[2]
        dz_err = 2.0 ** -11 * dD.double().abs() * (1.13 * (zr.abs() + 1) + 1.13)
        room = float((dz_err @ B.double().abs() * E.abs()).sum() + 2.0 ** -11 * (dA.double().abs() * E.abs()).sum() + (dz_err.sum(0) * e.abs()).sum())
        assert abs(got - slope) <= room + 1e-6 * abs(slope) + 1e-5


# ---- gated projections ---------------------------------------------------------------------------------

def _gated_case(M, F, K, dtype, transw, act, save, seed=0, pad=0, offset=0):
    g = _gen(seed)
    X = _draw(g, M, K, dtype, 1.0, False, pad, offset)
    Wg, Wu = (_draw(g, *((F, K) if transw else (K, F)), dtype, K ** -0.5, False, pad, offset) for _ in range(2))
    H = _out(M, F, dtype, pad, offset)
    G, U = (_out(M, F, dtype, pad, offset), _out(M, F, dtype, pad, offset)) if save else (None, None)
    dg.hgemm_gated(X, Wg, Wu, H, act=act, gate=G, up=U, transw=transw)
    _ok()
    want = ref.gated(X, Wg, Wu, act, transw)
    for name, out in (("H", H), ("G", G), ("U", U)):
        if out is not None:
            assert _padding_intact(out)
            ref.assert_within(out, *want[name], name)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("transw", [False, True])
@pytest.mark.parametrize("shape", [(1, 1, 1), (1, 64, 64), (4, 200, 1000), (16, 65, 70), (17, 63, 130), (33, 129, 200), (65, 500, 64),
                                   (129, 257, 65), (300, 260, 200), (1000, 777, 515)])
def test_gated(shape, transw, dtype):
    _gated_case(*shape, dtype, transw, ref.SILU, True, seed=sum(shape))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("transw", [False, True])
@pytest.mark.parametrize("pad,offset", [(0, 0), (3, 0), (0, 1)])
@pytest.mark.parametrize("shape", [(1, 3100, 130), (2, 4096, 515), (4, 3001, 300), (3, 40, 9000)])
def test_gated_of_few_rows(shape, pad, offset, transw, dtype):
    _gated_case(*shape, dtype, transw, ref.SILU, True, seed=sum(shape), pad=pad, offset=offset)
    _gated_case(*shape, dtype, transw, ref.GELU, False, seed=2, pad=pad, offset=offset)


@pytest.mark.parametrize("act", ref.ACTS)
@pytest.mark.parametrize("save", [False, True])
def test_gated_activations(act, save):
    _gated_case(3, 300, 200, torch.bfloat16, True, act, save, seed=act)
    _gated_case(300, 200, 100, torch.float16, False, act, save, seed=act)


@pytest.mark.parametrize("pad,offset", [(8, 0), (3, 0), (0, 1), (5, 4)])
@pytest.mark.parametrize("transw", [False, True])
def test_gated_strides_and_alignment(transw, pad, offset):
    _gated_case(7, 200, 136, torch.float16, transw, ref.SILU, True, seed=1, pad=pad, offset=offset)
    _gated_case(270, 136, 200, torch.bfloat16, transw, ref.GELU_TANH, True, seed=1, pad=pad, offset=offset)


@pytest.mark.parametrize("shape", [(4, 8192, 4096), (100, 512, 8192), (520, 1024, 4096), (4097, 1024, 512)])
def test_gated_large(shape):
    _gated_case(*shape, torch.bfloat16, True, ref.SILU, True, seed=3)


def _gated_grad_case(M, F, K, dtype, transw, act, seed=0, pad=0, offset=0, want=("dX", "dWg", "dWu")):
    g = _gen(seed)
    X = _draw(g, M, K, dtype, 1.0, False, pad, offset)
    Wg, Wu = (_draw(g, *((F, K) if transw else (K, F)), dtype, K ** -0.5, False, pad, offset) for _ in range(2))
    G, U, dH = (_draw(g, M, F, dtype, s, False, pad, offset) for s in (1.2, 1.0, 0.2))
    out = {"dX": _out(M, K, dtype, pad, offset), "dWg": _out(*Wg.shape, dtype, pad, offset), "dWu": _out(*Wu.shape, dtype, pad, offset)}
    dg.hgemm_gated_bwd(X, Wg, Wu, G, U, dH, act=act, transw=transw, **{k: v for k, v in out.items() if k in want})
    _ok()
    for name, (v, bound) in ref.gated_grad(X, Wg, Wu, G, U, dH, act, transw).items():
        if name not in want:
            assert bool(torch.isnan(out[name]).all())
            continue
        assert _padding_intact(out[name])
        ref.assert_within(out[name], v, bound, name)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("transw", [False, True])
@pytest.mark.parametrize("shape", [(1, 1, 1), (1, 130, 200), (5, 63, 65), (70, 200, 129), (300, 130, 260), (333, 1537, 1000)])
def test_gated_gradients(shape, transw, dtype):
    _gated_grad_case(*shape, dtype, transw, ref.SILU, seed=sum(shape))


@pytest.mark.parametrize("act", ref.ACTS)
def test_gated_gradients_activations(act):
    _gated_grad_case(90, 200, 136, torch.float16, True, act, seed=act)


@pytest.mark.parametrize("want", [("dX",), ("dWg",), ("dWu",), ("dWg", "dWu")])
def test_gated_gradients_optional_outputs(want):
    _gated_grad_case(150, 200, 96, torch.bfloat16, False, ref.GELU, seed=4, want=want)


@pytest.mark.parametrize("pad,offset", [(8, 0), (3, 0), (0, 1), (5, 4)])
@pytest.mark.parametrize("transw", [False, True])
def test_gated_gradients_strides_and_alignment(transw, pad, offset):
    _gated_grad_case(70, 136, 200, torch.float16, transw, ref.SILU, seed=6, pad=pad, offset=offset)


def test_gated_gradients_large():
    _gated_grad_case(2048, 4096, 1024, torch.bfloat16, True, ref.SILU, seed=2)


@pytest.mark.parametrize("transw", [False, True])
@pytest.mark.parametrize("shape", [(1, 1485, 1312), (12, 2408, 1874), (130, 3100, 200), (700, 130, 2600)])
def test_gradients_of_unlike_contractions_share_a_launch(shape, transw):
    """Few long sums beside many tiles of one or two k-blocks, and the other way round: spans that hold several tiles."""
    M, F, K = shape
    _gated_grad_case(M, F, K, torch.bfloat16, transw, ref.SILU, seed=M)
    _linear_grad_case(M, F, K, torch.float16, False, transw, ref.GELU_TANH, seed=M)
    _linear_grad_case(M, F, K, torch.float16, True, transw, ref.RELU, seed=M, integer=True, pad=3)


@pytest.mark.parametrize("N", [1, 8, 9, 63, 64, 65, 130, 520])
@pytest.mark.parametrize("M", [1, 31, 600, 9000])
def test_bias_gradient_over_strips_and_chunks(M, N):
    _linear_grad_case(M, N, 16, torch.bfloat16, False, True, ref.RELU, seed=N, integer=True, want=("dA", "dbias"))
    _linear_grad_case(M, N, 16, torch.float16, False, True, ref.SILU, seed=N, want=("dbias",), pad=1)


# ---- streams, refusals, abort path -----------------------------------------------------------------------

def test_calls_on_several_streams_do_not_share_scratch():
    """Cut tiles (workspace, counters) and packed operands in flight on four streams at once."""
    g = _gen(12)
    M, N, K = 20, 1001, 8000
    A, B = _draw(g, M, K, torch.bfloat16, 1.0, True, 3), _draw(g, N, K, torch.bfloat16, 1.0, True, 1)
    want = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    dg.hgemm_epilogue(A, B, want, transb=True)
    assert torch.equal(want, (A.double() @ B.double().t()).to(torch.bfloat16))
    streams = [torch.cuda.Stream() for _ in range(4)]
    outs = [[torch.empty_like(want) for _ in range(8)] for _ in streams]
    torch.cuda.synchronize()
    for i in range(8):
        for s, o in zip(streams, outs):
            with torch.cuda.stream(s):
                dg.hgemm_epilogue(A, B, o[i], transb=True)
    for s in streams:
        assert dg.hgemm_last_device_status(s) == dg.DGEMM_OK
    for o in outs:
        for d in o:
            assert torch.equal(d, want)


def test_captured_into_a_graph():
    g = _gen(13)
    A, B = _draw(g, 8, 4096, torch.bfloat16, 1.0, True), _draw(g, 512, 4096, torch.bfloat16, 1.0, True)
    D = torch.zeros(8, 512, dtype=torch.bfloat16, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        dg.hgemm_epilogue(A, B, D, transb=True)   # first call: allocates outside the capture
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        dg.hgemm_epilogue(A, B, D, transb=True)
    for _ in range(3):
        D.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(D, (A.double() @ B.double().t()).to(torch.bfloat16))


def test_binding_refuses_what_it_cannot_express():
    bf = torch.bfloat16
    A, B, D = (torch.zeros(*s, dtype=bf, device="cuda") for s in ((4, 8), (8, 6), (4, 6)))
    with pytest.raises(ValueError):
        dg.hgemm_epilogue(A, B, torch.zeros(4, 5, dtype=bf, device="cuda"))
    with pytest.raises(ValueError):
        dg.hgemm_epilogue(A.cpu(), B, D)
    with pytest.raises(ValueError):
        dg.hgemm_epilogue(A, torch.zeros(6, 8, dtype=bf, device="cuda").t(), D)      # columns not contiguous
    with pytest.raises(ValueError):
        dg.hgemm_epilogue(torch.zeros(1, 8, dtype=bf, device="cuda").expand(4, 8), B, D)
    with pytest.raises(TypeError):
        dg.hgemm_epilogue(A, B.half(), D)
    with pytest.raises(TypeError):
        dg.hgemm_epilogue(A.int(), B, D)
    with pytest.raises(ValueError):
        dg.hgemm_epilogue(A, B, D, bias=torch.zeros(5, dtype=bf, device="cuda"))
    for call in (lambda: dg.hgemm_epilogue(A.float(), B.float(), D.float()),          # binary32 operands
                 lambda: dg.hgemm_epilogue(A, B, D, act=9),
                 lambda: dg.hgemm_epilogue(A, B, D, preact=D),
                 lambda: dg.hgemm_gated(A, B, B, D, gate=torch.zeros_like(D)),        # gate without up
                 lambda: dg.hgemm_epilogue_bwd(A, B, D, act=dg.HGEMM_ACT_SILU, dA=torch.zeros_like(A))):  # no pre-activation
        with pytest.raises(dg.DgemmError):
            call()
    _ok()


@pytest.mark.parametrize("shape,gated", [((8, 300, 2000), False), ((600, 700, 500), False), ((4, 200, 3000), True), ((300, 300, 300), True)])
def test_dropped_loads_end_in_a_reported_timeout(shape, gated):
    """The producers skip their copies (nothing faults or spins without a limit): the call reports the
    timeout through the status word, and the next call is correct."""
    M, N, K = shape
    g = _gen(14)
    bf = torch.bfloat16
    A, B, C = _draw(g, M, K, bf, 1.0, True), _draw(g, N, K, bf, 1.0, True), _draw(g, N, K, bf, 1.0, True)
    D = _out(M, N, bf)

    def call():
        return dg.hgemm_gated(A, B, C, D, act=dg.HGEMM_ACT_NONE, transw=True) if gated else dg.hgemm_epilogue(A, B, D, transb=True)

    _ok()
    dg.hgemm_set_test_drop_loads(3000)
    try:
        assert call() == dg.DGEMM_OK
        assert dg.hgemm_last_device_status() == dg.binding.DGEMM_ERR_TIMEOUT
        assert dg.hgemm_last_device_status() == dg.DGEMM_OK
    finally:
        dg.hgemm_set_test_drop_loads(0)
    call()
    _ok()
    want = A.double() @ B.double().t()
    if gated:
        want = want * (A.double() @ C.double().t())
    assert torch.equal(D, want.to(bf))
