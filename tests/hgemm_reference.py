"""Plain 64-bit forms of the 16-bit products, the gated projections and layer norm, and the error
bounds the tests hold the kernels to. Independent of the library; works on any device.

Bounds. u is the unit roundoff of the output type, 2^-p for p significant bits: rounding to nearest is
off by at most u times the value (bfloat16 p = 8, binary16 p = 11, binary32 p = 24); tiny is half its
smallest subnormal step. A sum of
K products accumulated in binary32 is off by at most (K + 4) 2^-22 (|A||B|)_ij: each of the K additions
errs by one unit of the running sum (2^-23, truncation allowed), doubled for the alignment inside one
matrix instruction. The activations are 1.13-Lipschitz (gelu, silu: largest slope 1.13 and 1.10) and
evaluated within 2^-19 of their argument's size. One rounding to the output type follows.
"""
import math

import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24, torch.float64: 2.0 ** -53}
TINY = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -150, torch.float64: 0.0}
NONE, RELU, GELU, GELU_TANH, SILU = range(5)
ACTS = [NONE, RELU, GELU, GELU_TANH, SILU]
SLOPE = 1.13


def act(z, kind):
    if kind == NONE:
        return z
    if kind == RELU:
        return z.clamp_min(0)
    if kind == GELU:
        return 0.5 * z * (1 + torch.erf(z / math.sqrt(2)))
    if kind == GELU_TANH:
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    return z / (1 + torch.exp(-z))


def act_grad(z, kind):
    if kind == NONE:
        return torch.ones_like(z)
    if kind == RELU:
        return (z > 0).to(z.dtype)
    if kind == GELU:
        return 0.5 * (1 + torch.erf(z / math.sqrt(2))) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if kind == GELU_TANH:
        c = math.sqrt(2 / math.pi)
        t = torch.tanh(c * (z + 0.044715 * z ** 3))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z)
    s = 1 / (1 + torch.exp(-z))
    return s * (1 + z * (1 - s))


def op(x, trans):
    x = x.double()
    return x.t() if trans else x


def sum_error(K, absolute):
    return (K + 4) * 2.0 ** -22 * absolute


def rounded(want, err, dtype):
    """Bound of a value known within `err` after one rounding to `dtype`."""
    return err + U[dtype] * (want.abs() + err) * (1 + 2.0 ** -8) + TINY[dtype]


def linear(A, B, bias, kind, R, transa, transb):
    """(D, bound of D, Z, bound of Z) in 64 bits."""
    a, b = op(A, transa), op(B, transb)
    K = a.shape[1]
    z, size = a @ b, a.abs() @ b.abs()
    if bias is not None:
        z, size = z + bias.double(), size + bias.double().abs()
    zerr = sum_error(K, size)
    d = act(z, kind)
    derr = zerr if kind == NONE else SLOPE * zerr + 2.0 ** -19 * z.abs()
    if R is not None:
        d = d + R.double()
        derr = derr + 2.0 ** -23 * (d.abs() + R.double().abs())
    return d, rounded(d, derr, A.dtype), z, rounded(z, zerr, A.dtype)


def linear_grad(A, B, Z, kind, dD, transa, transb):
    """{name: (value, bound)} of dA, dB, dbias in 64 bits. dZ is rounded to 16 bits before the products: every
    term of a sum is off by u (and the 2^-19 of the derivative)."""
    t = A.dtype
    a, b = op(A, transa), op(B, transb)
    dz = dD.double() if kind == NONE else dD.double() * act_grad(Z.double(), kind)
    rough = 0.0 if kind == NONE else 2.0 ** -20
    dz_err = (0.0 if kind == NONE else U[t] * (1 + 2.0 ** -8)) * dz.abs() + rough * dD.double().abs() + (0.0 if kind == NONE else TINY[t])
    out = {}
    for name, l, r, le, re, trans in (("dA", dz, b.t(), dz_err, None, transa), ("dB", a.t(), dz, None, dz_err, transb)):
        v = l @ r
        err = sum_error(l.shape[1], l.abs() @ r.abs()) + (le @ r.abs() if le is not None else l.abs() @ re)
        bound = rounded(v, err, t)
        out[name] = (v.t(), bound.t()) if trans else (v, bound)
    M = dz.shape[0]
    out["dbias"] = (dz.sum(0), ((M + 2) * 2.0 ** -23 + 2.0 ** -22) * dz.abs().sum(0) + rough * dD.double().abs().sum(0) + 1e-38)
    return out


def gated(X, Wg, Wu, kind, transw):
    x, wg, wu = X.double(), op(Wg, transw), op(Wu, transw)
    K = x.shape[1]
    g, u = x @ wg, x @ wu
    ge, ue = sum_error(K, x.abs() @ wg.abs()), sum_error(K, x.abs() @ wu.abs())
    f = act(g, kind)
    fe = SLOPE * ge + 2.0 ** -19 * g.abs()
    h = f * u
    he = f.abs() * ue + u.abs() * fe + fe * ue + 2.0 ** -23 * h.abs()
    return {"H": (h, rounded(h, he, X.dtype)), "G": (g, rounded(g, ge, X.dtype)), "U": (u, rounded(u, ue, X.dtype))}


def gated_grad(X, Wg, Wu, G, Up, dH, kind, transw):
    t = X.dtype
    x, wg, wu = X.double(), op(Wg, transw), op(Wu, transw)
    g, u, dh = G.double(), Up.double(), dH.double()
    dg, du = dh * u * act_grad(g, kind), dh * act(g, kind)
    ge = U[t] * (1 + 2.0 ** -8) * dg.abs() + 2.0 ** -20 * (dh * u).abs() + TINY[t]
    ue = U[t] * (1 + 2.0 ** -8) * du.abs() + 2.0 ** -20 * (dh * g).abs() + TINY[t]
    dx = dg @ wg.t() + du @ wu.t()
    size = dg.abs() @ wg.abs().t() + du.abs() @ wu.abs().t()
    xe = sum_error(2 * g.shape[1], size) + ge @ wg.abs().t() + ue @ wu.abs().t()
    out = {"dX": (dx, rounded(dx, xe, t))}
    for name, d, e in (("dWg", dg, ge), ("dWu", du, ue)):
        v = x.t() @ d
        bound = rounded(v, sum_error(x.shape[0], x.abs().t() @ d.abs()) + x.abs().t() @ e, t)
        out[name] = (v.t(), bound.t()) if transw else (v, bound)
    return out


def norm(X, gamma, beta, eps):
    """(y, bound, mean, bound, rstd, bound). A sum of n binary32 terms errs by (log2-shaped or not) at most
    n 2^-24 of the sum of absolute values; the kernels add in at most 64 + 32 sequential steps, and the
    bound below allows 256."""
    x = X.double()
    n = x.shape[1]
    steps = 256 * 2.0 ** -24
    mean = x.mean(1, keepdim=True)
    me = steps * x.abs().mean(1, keepdim=True) + 1e-38
    d = x - mean
    var = (d * d).mean(1, keepdim=True)
    ve = 2 * steps * var + 2 * me * d.abs().mean(1, keepdim=True) + me * me
    rstd = (var + eps).rsqrt()
    # |d rstd| = rstd^3 / 2 |d var|, over the interval the variance can lie in
    low = (var - ve).clamp_min(0) + eps
    re = 0.5 * ve * rstd * rstd * low.clamp_min(1e-300).rsqrt() + 2.0 ** -22 * rstd
    xh = d * rstd
    xe = me * rstd + d.abs() * re + me * re + 2.0 ** -22 * xh.abs()
    w = torch.ones(n, dtype=torch.float64, device=x.device) if gamma is None else gamma.double()
    b = torch.zeros(n, dtype=torch.float64, device=x.device) if beta is None else beta.double()
    y = xh * w + b
    ye = xe * w.abs() + 2.0 ** -22 * (xh * w).abs() + 2.0 ** -23 * y.abs()
    return y, rounded(y, ye, X.dtype), mean[:, 0], me[:, 0], rstd[:, 0], re[:, 0]


def norm_grad(X, gamma, mean, rstd, dY):
    x, dy = X.double(), dY.double()
    n = x.shape[1]
    m, r = mean.double()[:, None], rstd.double()[:, None]
    xh = (x - m) * r
    xe = 2.0 ** -22 * ((x.abs() + m.abs()) * r)
    w = dy if gamma is None else dy * gamma.double()
    steps = 256 * 2.0 ** -24
    s1, s2 = w.mean(1, keepdim=True), (w * xh).mean(1, keepdim=True)
    e1 = steps * w.abs().mean(1, keepdim=True)
    e2 = steps * (w * xh).abs().mean(1, keepdim=True) + (w.abs() * xe).mean(1, keepdim=True)
    dx = r * (w - s1 - xh * s2)
    de = r * (e1 + xh.abs() * e2 + xe * s2.abs() + 2.0 ** -22 * (w.abs() + s1.abs() + (xh * s2).abs()))
    rows = x.shape[0]
    param = (rows + 16) * 2.0 ** -23
    return {"dx": (dx, rounded(dx, de, X.dtype)),
            "dgamma": ((dy * xh).sum(0), param * (dy * xh).abs().sum(0) + (dy.abs() * xe).sum(0) + 1e-38),
            "dbeta": (dy.sum(0), param * dy.abs().sum(0) + 1e-38)}


def assert_within(got, want, bound, what):
    got = got.double()
    bad = ~((got - want).abs() <= bound)
    if bool(bad.any()):
        ratio = ((got - want).abs() / bound.clamp_min(1e-300))
        ratio = torch.where(torch.isfinite(ratio), ratio, torch.full_like(ratio, 1e30))
        at = int(ratio.argmax())
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} values out of bounds, worst {float(ratio.max()):.3g} times at flat "
                             f"index {at}: got {float(got.reshape(-1)[at]):.6g}, want {float(want.reshape(-1)[at]):.6g}")
