"""Gradients in binary16 whose element-wise part (dZ, dG, dU) lies outside binary16's range while the results lie inside it,
and beside infinities and NaN. Needs a B200.

Bounds. As in ``hgemm_reference``, but the element-wise part may be scaled by a power of two before it is rounded, so that its
smallest step, 2^-25 at the scale at which the largest value is 2^14 or more, is 2^-39 of the largest value. Where the part is
left as it is (its largest value from 2^-4 to 65504), the step is 2^-25 absolute."""
import pytest
import torch

import hgemm_reference as ref
import paper_2003_00532_b200 as dg
from test_gpu_hgemm import _draw, _gen, _ok, _out, _padding_intact

pytestmark = pytest.mark.gpu

H = torch.float16


def _step(*parts):
    top = max(float(p.abs().max()) for p in parts)
    return 2.0 ** -25 if 2.0 ** -4 <= top < 65520 else 2.0 ** -39 * top


def _gated_bounds(X, Wg, Wu, G, Up, dH, kind, transw):
    x, wg, wu = X.double(), ref.op(Wg, transw), ref.op(Wu, transw)
    g, u, dh = G.double(), Up.double(), dH.double()
    dg_, du = dh * u * ref.act_grad(g, kind), dh * ref.act(g, kind)
    step = _step(dg_, du)
    ge = ref.U[H] * (1 + 2.0 ** -8) * dg_.abs() + 2.0 ** -20 * (dh * u).abs() + step
    ue = ref.U[H] * (1 + 2.0 ** -8) * du.abs() + 2.0 ** -20 * (dh * g).abs() + step
    dx = dg_ @ wg.t() + du @ wu.t()
    size = dg_.abs() @ wg.abs().t() + du.abs() @ wu.abs().t()
    out = {"dX": (dx, ref.rounded(dx, ref.sum_error(2 * g.shape[1], size) + ge @ wg.abs().t() + ue @ wu.abs().t(), H))}
    for name, d, e in (("dWg", dg_, ge), ("dWu", du, ue)):
        v = x.t() @ d
        bound = ref.rounded(v, ref.sum_error(x.shape[0], x.abs().t() @ d.abs()) + x.abs().t() @ e, H)
        out[name] = (v.t(), bound.t()) if transw else (v, bound)
    return out, max(float(dg_.abs().max()), float(du.abs().max()))


def _linear_bounds(A, B, Z, kind, dD, transa, transb):
    a, b, dd = ref.op(A, transa), ref.op(B, transb), dD.double()
    dz = dd * ref.act_grad(Z.double(), kind)
    e = ref.U[H] * (1 + 2.0 ** -8) * dz.abs() + 2.0 ** -20 * dd.abs() + _step(dz)
    out = {}
    for name, l, r, err, trans in (("dA", dz, b.t(), e @ b.t().abs(), transa), ("dB", a.t(), dz, a.t().abs() @ e, transb)):
        v = l @ r
        bound = ref.rounded(v, ref.sum_error(l.shape[1], l.abs() @ r.abs()) + err, H)
        out[name] = (v.t(), bound.t()) if trans else (v, bound)
    M = dz.shape[0]
    out["dbias"] = (dz.sum(0), ((M + 2) * 2.0 ** -23 + 2.0 ** -22) * dz.abs().sum(0) + 2.0 ** -20 * dd.abs().sum(0) + 1e-38)
    return out, float(dz.abs().max())


def _gated(M, F, K, kind, transw, dh, up, gate, weight, x, seed=0, pad=0):
    g = _gen(seed)
    X = _draw(g, M, K, H, x, pad=pad)
    Wg, Wu = (_draw(g, *((F, K) if transw else (K, F)), H, weight, pad=pad) for _ in range(2))
    G, U, dH = (_draw(g, M, F, H, s, pad=pad) for s in (gate, up, dh))
    out = {"dX": _out(M, K, H, pad), "dWg": _out(*Wg.shape, H, pad), "dWu": _out(*Wu.shape, H, pad)}
    dg.hgemm_gated_bwd(X, Wg, Wu, G, U, dH, act=kind, transw=transw, **out)
    _ok()
    want, top = _gated_bounds(X, Wg, Wu, G, U, dH, kind, transw)
    for name, (v, bound) in want.items():
        assert float(v.abs().max()) < 65504 and _padding_intact(out[name])
        ref.assert_within(out[name], v, bound, name)
    return top


def _linear(M, N, K, kind, transa, transb, dd, weight, a, seed=0, pad=0, z=1.5):
    g = _gen(seed)
    A = _draw(g, *((K, M) if transa else (M, K)), H, a, pad=pad)
    B = _draw(g, *((N, K) if transb else (K, N)), H, weight, pad=pad)
    Z = _draw(g, M, N, H, z, pad=pad)
    dD = _draw(g, M, N, H, 1.0, pad=pad)
    dD.copy_((dD.float().clamp(-1, 1) * dd).to(H))
    out = {"dA": _out(*A.shape, H, pad), "dB": _out(*B.shape, H, pad), "dbias": torch.full((N,), float("nan"), device="cuda")}
    dg.hgemm_epilogue_bwd(A, B, dD, act=kind, preact=Z, transa=transa, transb=transb, **out)
    _ok()
    want, top = _linear_bounds(A, B, Z, kind, dD, transa, transb)
    for name, (v, bound) in want.items():
        ref.assert_within(out[name], v, bound, name)
    return top


SHAPES = [(1, 70, 130), (37, 65, 64), (130, 257, 96), (700, 520, 264)]


@pytest.mark.parametrize("transw", [False, True])
@pytest.mark.parametrize("pad", [0, 3])
@pytest.mark.parametrize("shape", SHAPES)
def test_gated_parts_above_the_range(shape, pad, transw):
    """Loss-scaled gradients: |dH U| well above 65504, weights and inputs that bring the results back."""
    top = _gated(*shape, ref.SILU, transw, dh=3000.0, up=50.0, gate=4.0, weight=2.0 ** -10, x=2.0 ** -10, seed=sum(shape), pad=pad)
    assert top > 65504


@pytest.mark.parametrize("transw", [False, True])
@pytest.mark.parametrize("shape", SHAPES)
def test_gated_parts_below_the_range(shape, transw):
    """Gradients without loss scaling: every dH U below binary16's smallest number, large weights and inputs."""
    top = _gated(*shape, ref.GELU_TANH, transw, dh=2.0 ** -16, up=2.0 ** -10, gate=2.0 ** -10, weight=2.0 ** 9, x=2.0 ** 9, seed=sum(shape))
    assert top < 2.0 ** -22


@pytest.mark.parametrize("kind", [ref.NONE, ref.RELU, ref.GELU, ref.SILU])
def test_gated_parts_of_every_activation(kind):
    assert _gated(90, 200, 136, kind, True, dh=3000.0, up=50.0, gate=40.0, weight=2.0 ** -10, x=2.0 ** -10, seed=kind) > 65504
    assert _gated(90, 200, 136, kind, True, dh=2.0 ** -14, up=2.0 ** -8, gate=2.0 ** -8, weight=2.0 ** 8, x=2.0 ** 8, seed=kind) < 2.0 ** -16


@pytest.mark.parametrize("kind", [ref.GELU, ref.GELU_TANH, ref.SILU])
@pytest.mark.parametrize("transa,transb", [(False, True), (False, False), (True, True)])
@pytest.mark.parametrize("shape", SHAPES)
def test_linear_parts_outside_the_range(shape, transa, transb, kind):
    top = _linear(*shape, kind, transa, transb, dd=65000.0, weight=2.0 ** -10, a=2.0 ** -10, seed=sum(shape))
    assert top > 60000
    assert _linear(*shape, kind, transa, transb, dd=2.0 ** -14, weight=2.0 ** 8, a=2.0 ** 8, seed=1, pad=3) < 2.0 ** -13


def test_linear_part_overflows_where_the_slope_is_above_one():
    assert _linear(300, 264, 96, ref.GELU, False, True, dd=65504.0, weight=2.0 ** -10, a=2.0 ** -10, seed=3) > 65520


def test_large_small_and_ordinary_parts_in_turn():
    """Nothing of one call's range is left for the next."""
    for i, (dh, w) in enumerate([(3000.0, -10), (0.2, 0), (2.0 ** -16, 8), (0.2, 0), (3000.0, -10), (2.0 ** -16, 8), (0.2, 0)]):
        up = 50.0 if dh > 1 else 1.0 if dh > 0.1 else 2.0 ** -8
        _gated(200, 136, 72, ref.SILU, True, dh=dh, up=up, gate=2.0, weight=2.0 ** w, x=2.0 ** w / 4, seed=i)


def test_all_parts_zero():
    X, W = torch.ones(40, 64, dtype=H, device="cuda"), torch.ones(96, 64, dtype=H, device="cuda")
    P, Z = torch.ones(40, 96, dtype=H, device="cuda"), torch.zeros(40, 96, dtype=H, device="cuda")
    dX, dW = _out(40, 64, H), _out(96, 64, H)
    dg.hgemm_gated_bwd(X, W, W, P, P, Z, dX=dX, dWg=dW, transw=True)
    assert bool((dX == 0).all()) and bool((dW == 0).all())
    dg.hgemm_epilogue_bwd(X, W, Z, act=ref.SILU, preact=P, dA=dX, dB=dW, transb=True)
    assert bool((dX == 0).all()) and bool((dW == 0).all())


@pytest.mark.parametrize("scale,weight", [(3000.0, 2.0 ** -10), (0.2, 0.1)])
def test_infinities_and_nan_do_not_change_the_scale_of_the_rest(scale, weight):
    """An infinity and a NaN in dH: their rows of dX and columns of dW are lost, everything else is as without them."""
    g = _gen(9)
    M, F, K = 150, 200, 72
    X, Wg, Wu = _draw(g, M, K, H, weight), _draw(g, F, K, H, weight), _draw(g, F, K, H, weight)
    G, U, dH = _draw(g, M, F, H, 2.0), _draw(g, M, F, H, 50.0 if scale > 1 else 1.0), _draw(g, M, F, H, scale)
    dH[3, 5], dH[77, 130] = 0.0, 0.0
    plain = {"dX": _out(M, K, H), "dWg": _out(F, K, H), "dWu": _out(F, K, H)}
    dg.hgemm_gated_bwd(X, Wg, Wu, G, U, dH, transw=True, **plain)
    dH[3, 5], dH[77, 130] = float("inf"), float("nan")
    out = {"dX": _out(M, K, H), "dWg": _out(F, K, H), "dWu": _out(F, K, H)}
    dg.hgemm_gated_bwd(X, Wg, Wu, G, U, dH, transw=True, **out)
    _ok()
    for name, rows in (("dX", (3, 77)), ("dWg", (5, 130)), ("dWu", (5, 130))):
        keep = torch.ones(out[name].shape[0], dtype=torch.bool, device="cuda")
        keep[list(rows)] = False
        assert not bool(torch.isfinite(out[name][~keep]).all())
        assert bool(torch.isfinite(out[name][keep]).all()) and torch.equal(out[name][keep], plain[name][keep]), name


def test_same_bits_every_time():
    first = None
    for _ in range(5):
        g = _gen(2)
        X, Wg, Wu = _draw(g, 300, 264, H, 2.0 ** -10), _draw(g, 700, 264, H, 2.0 ** -10), _draw(g, 700, 264, H, 2.0 ** -10)
        G, U, dH = _draw(g, 300, 700, H, 4.0), _draw(g, 300, 700, H, 50.0), _draw(g, 300, 700, H, 3000.0)
        out = [_out(300, 264, H), _out(700, 264, H), _out(700, 264, H)]
        dg.hgemm_gated_bwd(X, Wg, Wu, G, U, dH, dX=out[0], dWg=out[1], dWu=out[2], transw=True)
        first = out if first is None else first
        assert all(torch.equal(a, b) for a, b in zip(out, first))


def test_calls_on_several_streams_keep_their_own_scale():
    g = _gen(12)
    M, F, K = 200, 264, 136
    sets = []
    for i, (dh, up, w) in enumerate(((3000.0, 50.0, 2.0 ** -10), (0.2, 1.0, 0.1), (2.0 ** -16, 2.0 ** -8, 256.0), (3000.0, 50.0, 2.0 ** -10))):
        X, Wg, Wu = _draw(g, M, K, H, w), _draw(g, F, K, H, w), _draw(g, F, K, H, w)
        G, U, dH = _draw(g, M, F, H, 2.0), _draw(g, M, F, H, up), _draw(g, M, F, H, dh)
        want = _out(M, K, H)
        dg.hgemm_gated_bwd(X, Wg, Wu, G, U, dH, dX=want, transw=True)
        sets.append((torch.cuda.Stream(), (X, Wg, Wu, G, U, dH), want, [_out(M, K, H) for _ in range(8)]))
    torch.cuda.synchronize()
    for i in range(8):
        for s, args, _, outs in sets:
            with torch.cuda.stream(s):
                dg.hgemm_gated_bwd(*args, dX=outs[i], transw=True)
    for s, _, want, outs in sets:
        assert dg.hgemm_last_device_status(s) == dg.DGEMM_OK
        assert bool(torch.isfinite(want).all()) and all(torch.equal(o, want) for o in outs)
