"""Plain 64-bit forms of RMS norm, rows in 8 bits, dropout and the products of 8-bit operands, and the error bounds the tests hold the
kernels to (``hgemm_reference`` has u, tiny and the bounds of sums and activations). Independent of the library; works on any device.

Bounds. The sum s = x + r is one binary32 addition, off by 2^-24 |s|. A sum of n squares is off by the additions' roundings, at most
256 in a row (the kernels have at most 64), and two for each square: (256 + 4) 2^-24 of itself; rstd by half of that and 2^-22 for
the reciprocal root; y by those and three more roundings of 2^-24. Together VALUE = 2^-16 of its size, twice that allowed.

e4m3 has values m 2^(e - 3), e >= -6: rounding to nearest is off by at most half a step, 2^(e - 4) for a value of exponent e.
"""
import torch

import hgemm_reference as ref

VALUE = 2.0 ** -15
TOP = 448.0
LEAST = 2.0 ** -100
E4M3 = torch.float8_e4m3fn


def rms(X, R, gamma, eps):
    """(s, y, rstd) in 64 bits."""
    s = X.double() if R is None else X.double() + R.double()
    rstd = (s.square().mean(1) + eps).rsqrt()
    y = s * rstd[:, None]
    return s, y if gamma is None else y * gamma.double(), rstd


def value_bound(want, dtype):
    """Bound of a y that is known within VALUE of its size, after rounding to `dtype`."""
    return ref.rounded(want, VALUE * want.abs(), dtype)


def sum_bound(s, dtype):
    return ref.rounded(s, 2.0 ** -24 * s.abs(), dtype)


def half_step(v):
    """Half of e4m3's step at |v|."""
    e = torch.frexp(v.abs().clamp_min(2.0 ** -10))[1].double() - 1
    return torch.exp2(e.clamp_min(-6) - 4)


def assert_eight(Q, scale, y, value=VALUE):
    """Q and scale are the rows y in 8 bits, y known within `value` of its size."""
    want = y.abs().amax(1).clamp_min(LEAST) / TOP
    # the division and the multiplications by rstd: four roundings
    ref.assert_within(scale, want, (value + 2.0 ** -21) * want, "scale")
    v = y / scale.double()[:, None]
    # y / scale as the kernels take it errs by value + four roundings of its size; a rounding to nearest from there (the step of the
    # larger neighbour, if the error lifts it over a power of two)
    err = (value + 2.0 ** -21) * v.abs()
    ref.assert_within(Q, v, half_step(v.abs() + err) * (1 + 2.0 ** -20) + err, "Q")


def rms_grad(S, gamma, rstd, dY, dS):
    """{name: (value, bound)}; as the bounds of layer norm's gradients, with one sum."""
    s, dy, r = S.double(), dY.double(), rstd.double()[:, None]
    xh = s * r
    xe = 2.0 ** -23 * xh.abs()
    w = dy if gamma is None else dy * gamma.double()
    steps = 256 * 2.0 ** -24
    t = (w * xh).mean(1, keepdim=True)
    te = steps * (w * xh).abs().mean(1, keepdim=True) + (w.abs() * xe).mean(1, keepdim=True)
    dx = r * (w - xh * t)
    de = r * (xh.abs() * te + xe * t.abs() + 2.0 ** -22 * (w.abs() + (xh * t).abs()))
    if dS is not None:
        dx = dx + dS.double()
        de = de + 2.0 ** -23 * (dx.abs() + dS.double().abs())
    param = (s.shape[0] + 16) * 2.0 ** -23
    return {"dX": (dx, ref.rounded(dx, de, S.dtype)),
            "dgamma": ((dy * xh).sum(0), param * (dy * xh).abs().sum(0) + (dy.abs() * xe).sum(0) + 1e-38)}


def philox(c, k):
    """Philox4x32-10 on Python integers: four counter words and two key words."""
    c, k = list(c), list(k)
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [b >> 32 ^ c[1] ^ k[0], b & 0xFFFFFFFF, a >> 32 ^ c[3] ^ k[1], a & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def words(rows, cols, seed, offset, device, first_row=0, first_col=0):
    """The random words of a matrix, or of a part of one that begins at a multiple of four columns."""
    low = 0xFFFFFFFF
    a = torch.arange(first_col // 4, first_col // 4 + (cols + 3) // 4, dtype=torch.int64, device=device).expand(rows, -1)
    b = torch.arange(first_row, first_row + rows, dtype=torch.int64, device=device)[:, None].expand_as(a)
    c = [a, b, torch.full_like(a, offset & low), torch.full_like(a, offset >> 32 & low)]
    k = [seed & low, seed >> 32 & low]
    for _ in range(10):
        x, y = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(y >> 32 & low) ^ c[1] ^ k[0], y & low, (x >> 32 & low) ^ c[3] ^ k[1], x & low]
        k = [(k[0] + 0x9E3779B9) & low, (k[1] + 0xBB67AE85) & low]
    return torch.stack(c, 2).reshape(rows, -1)[:, :cols]


def dropout(X, R, p, seed, offset):
    """(y, bound): 1 / (1 - p) in binary32, the product and the sum are off by 2^-24 each."""
    keep = words(*X.shape, seed, offset, X.device) >= int(p * 2.0 ** 32 + 0.5)
    x = torch.where(keep, X.double() / (1 - p) if p < 1 else X.double(), torch.zeros((), dtype=torch.float64, device=X.device))
    y = x if R is None else x + R.double()
    return y, ref.rounded(y, 2.0 ** -22 * x.abs() + 2.0 ** -23 * y.abs(), X.dtype), keep


def _scaled(q, scale):
    return q.double() if scale is None else q.double() * scale.double()[:, None]


def linear8(A, B, sa, sb, bias, kind, R, dtype):
    """(D, bound, Z, bound): the bounds of the 16-bit products, and 2^-22 for the two scales."""
    a, b = _scaled(A, sa), _scaled(B, sb)
    z, size = a @ b.t(), a.abs() @ b.abs().t()
    zerr = ref.sum_error(a.shape[1], size) + 2.0 ** -22 * z.abs()
    if bias is not None:
        z = z + bias.double()
        zerr = zerr + 2.0 ** -23 * (z.abs() + bias.double().abs())
    d = ref.act(z, kind)
    derr = zerr if kind == ref.NONE else ref.SLOPE * zerr + 2.0 ** -19 * z.abs()
    if R is not None:
        d = d + R.double()
        derr = derr + 2.0 ** -23 * (d.abs() + R.double().abs())
    return d, ref.rounded(d, derr, dtype), z, ref.rounded(z, zerr, dtype)


def gated8(X, Wg, Wu, sx, sg, su, kind, dtype):
    x, wg, wu = _scaled(X, sx), _scaled(Wg, sg), _scaled(Wu, su)
    g, u = x @ wg.t(), x @ wu.t()
    K = x.shape[1]
    ge = ref.sum_error(K, x.abs() @ wg.abs().t()) + 2.0 ** -22 * g.abs()
    ue = ref.sum_error(K, x.abs() @ wu.abs().t()) + 2.0 ** -22 * u.abs()
    f = ref.act(g, kind)
    fe = ref.SLOPE * ge + 2.0 ** -19 * g.abs()
    h = f * u
    he = f.abs() * ue + u.abs() * fe + fe * ue + 2.0 ** -23 * h.abs()
    return {"H": (h, ref.rounded(h, he, dtype)), "G": (g, ref.rounded(g, ge, dtype)), "U": (u, ref.rounded(u, ue, dtype))}
