"""More operators of a transformer's feed-forward path, as cases that can be measured: root-mean-square norm with the residual's
addition (16- and 32-bit output, or 8 bits with a scale per row), its backward pass, rows brought to 8 bits, the matrix product and
the gated projections of 8-bit operands with their scales, and dropout with the residual's addition.

``listed`` names fixed cases, ``draw`` makes more of the same ranges. ``prepare`` makes what a program has in hand before a call,
``run`` makes one pass: with ``own`` false in elementary 32-bit torch operations, with ``own`` true through
``paper_2003_00532_b200``. ``exact`` computes the same outputs in 64 bits. Matrices are row-major; ``pad`` elements are added to
every leading dimension. 8-bit values are e4m3 (``torch.float8_e4m3fn``) and returned as such, next to their scales.
"""
import math

import numpy as np
import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_BYTES = {"bf16": 2, "f16": 2, "f32": 4}
_E4M3 = torch.float8_e4m3fn
_TOP = 448.0          # largest e4m3 value
_LEAST = 2.0 ** -100  # rows that are smaller than this are scaled as if it were their largest value
_EPS = 1e-5
_MOST_FLOPS = 2.0 * 8192 * 4096 * 8192


def listed():
    return [
        # Residual addition and norm of one new token: the smallest call, latency alone.
        _norm("rms_token", "rms", "bf16", 1, 4096, res=True),
        # The same of a training batch or a long prompt, sum and statistics kept for the backward pass: memory.
        _norm("rms_batch", "rms", "bf16", 8192, 4096, res=True),
        # Its backward pass: the residual stream's gradient joins, the weight's gradient is summed over all rows.
        _norm("rms_grad", "rms_grad", "bf16", 8192, 4096, res=True),
        # The same in single precision on the library's ragged row length: rows that are not 16-byte aligned.
        _norm("rms_grad_ragged", "rms_grad", "f32", 4097, 1537, res=False),
        # The new tokens of 16 requests on their way into 8-bit products: latency, two reductions in a row.
        _norm("rms8_tokens", "rms8", "bf16", 16, 8192, res=True),
        # A ragged prompt in half precision on the same way: memory.
        _norm("rms8_batch", "rms8", "f16", 4097, 8192, res=True),
        # Hidden activations between two 8-bit products, at the library's 2088-row configuration.
        _norm("rows8_batch", "rows8", "bf16", 2088, 8192, res=False),
        # Output projection of one new token with 8-bit weights, bias and residual: reading 4096 x 4096 bytes.
        _linear8("linear8_token", "bf16", 1, 4096, 4096, act="none", bias=True, res=True, save=False),
        # A long prompt through 8-bit weights: compute-bound, the largest product.
        _linear8("linear8_batch", "bf16", 8192, 4096, 8192, act="gelu_tanh", bias=True, res=False, save=False),
        # Gate and up projections of a ragged prompt.
        _gated8("gated8_batch", "f16", 4097, 8192, 2048, act="silu", save=False),
        # Dropout of a sublayer's output and its addition to the residual stream, training batch.
        _dropout("dropout_batch", "dropout", "bf16", 8192, 4096, p=0.1, res=True),
        # The backward pass of a short ragged batch: odd sizes, rows of any alignment, the mask made again.
        _dropout("dropout_grad_ragged", "dropout_grad", "f16", 1000, 1537, p=0.25, res=False, pad=3),
    ]


def _case(name, c):
    return dict(c, name=name) if name else c


def _norm(name, op, dtype, rows, cols, *, res, pad=0):
    return _case(name, {"op": op, "dtype": dtype, "rows": rows, "cols": cols, "res": res, "pad": pad})


def _linear8(name, dtype, M, N, K, *, act, bias, res, save, pad=0):
    return _case(name, {"op": "linear8", "dtype": dtype, "M": M, "N": N, "K": K, "act": act, "bias": bias, "res": res, "save": save, "pad": pad})


def _gated8(name, dtype, M, F, K, *, act, save, pad=0):
    return _case(name, {"op": "gated8", "dtype": dtype, "M": M, "F": F, "K": K, "act": act, "save": save, "pad": pad})


def _dropout(name, op, dtype, rows, cols, *, p, res, pad=0):
    return _case(name, {"op": op, "dtype": dtype, "rows": rows, "cols": cols, "p": p, "res": res, "pad": pad})


def _size(rng, lo, hi):
    """Log-uniform in lo..hi; every other one brought to a multiple of 64 or 8, the rest as they fall."""
    n = math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))
    step = rng.choice([1, 1, 8, 64])
    return min(hi, max(lo, int(round(n / step)) * step))


def draw(rng):
    op = rng.choice(["rms", "rms", "rms_grad", "rms_grad", "rms8", "rms8", "rows8", "linear8", "linear8", "gated8", "gated8",
                     "dropout", "dropout_grad"])
    if op not in ("linear8", "gated8"):
        while True:
            rows, cols = _size(rng, 1, 16384), _size(rng, 32, 16384)
            if rows * cols <= 8192 * 4096:
                break
        dtype, pad, res = rng.choice(["bf16", "bf16", "f16", "f32"]), rng.choice([0, 0, 8, 3]), rng.random() < 0.7
        if op.startswith("dropout"):
            # 32-bit dropout of the largest size would cost more than the largest listed one
            return _dropout(None, op, "bf16" if dtype == "f32" and rows * cols > 4096 * 4096 else dtype, rows, cols,
                            p=rng.choice([0.05, 0.1, 0.2, 0.5]), res=res and op == "dropout", pad=pad)
        return _norm(None, op, dtype, rows, cols, res=res and op != "rows8", pad=pad)
    dtype, pad = rng.choice(["bf16", "f16"]), rng.choice([0, 0, 0, 16, 3])
    while True:
        M, N, K = _size(rng, 1, 8192), _size(rng, 64, 8192), _size(rng, 64, 8192)
        if 2.0 * M * N * K * (2 if op == "gated8" else 1) <= _MOST_FLOPS:
            break
    if op == "gated8":
        return _gated8(None, dtype, M, N, K, act=rng.choice(["silu", "gelu_tanh", "gelu"]), save=rng.random() < 0.3, pad=pad)
    act = rng.choice(["none", "relu", "gelu", "gelu_tanh", "silu"])
    return _linear8(None, dtype, M, N, K, act=act, bias=rng.random() < 0.7, res=rng.random() < 0.5, save=rng.random() < 0.3 and act != "none", pad=pad)


def work(case):
    e, op = _BYTES[case["dtype"]], case["op"]
    if op == "linear8":  # 8-bit operands, their scales and the bias in; 16-bit matrices
        M, N, K = case["M"], case["N"], case["K"]
        return {"bytes": M * K + N * K + 4 * (M + N) + e * (M * N * (1 + case["res"] + case["save"]) + N * case["bias"]), "flops": 2 * M * N * K}
    if op == "gated8":
        M, F, K = case["M"], case["F"], case["K"]
        return {"bytes": M * K + 2 * F * K + 4 * (M + 2 * F) + e * M * F * (3 if case["save"] else 1), "flops": 4 * M * F * K}
    r, c = case["rows"], case["cols"]
    n, res = r * c, case["res"]
    if op == "rms":  # x, r, gamma in; s (with a residual), y, rstd out
        return {"bytes": e * (n * (2 + 2 * res) + c) + 4 * r, "flops": 5 * n}
    if op == "rms_grad":  # s, dy, ds, gamma, rstd in; dx, dgamma out
        return {"bytes": e * (n * (3 + res) + c) + 4 * r + 4 * c, "flops": 9 * n}
    if op == "rms8":  # x, r, gamma in; s, the 8-bit values and their scales out
        return {"bytes": e * (n * (1 + 2 * res) + c) + n + 4 * r, "flops": 7 * n}
    if op == "rows8":
        return {"bytes": e * n + n + 4 * r, "flops": 2 * n}
    return {"bytes": e * n * (2 + res), "flops": 20 * n}  # x, r in; y out


# ---- inputs ---------------------------------------------------------------------------------------

def _new(rows, cols, pad, t):
    return torch.empty(rows, cols + pad, dtype=t, device="cuda")[:, :cols]


def _normal(g, rows, cols, pad, t, scale):
    x = _new(rows, cols, pad, t)
    x.copy_(torch.randn(rows, cols, device="cuda", generator=g) * scale)
    return x


def _stream(g, rows, cols, pad, t):
    """The residual stream: rows of different size."""
    x = _new(rows, cols, pad, t)
    x.copy_(torch.randn(rows, cols, device="cuda", generator=g) * (0.5 + 2 * torch.rand(rows, 1, device="cuda", generator=g)))
    return x


def _eight(g, rows, cols, pad, scale):
    """An 8-bit matrix with a scale per row, as weights and activations are brought to 8 bits."""
    x = _stream(g, rows, cols, 0, torch.float32) * scale
    top = x.abs().amax(1, keepdim=True) / _TOP
    q = _new(rows, cols, pad, _E4M3)
    q.copy_((x / top).clamp(-_TOP, _TOP).to(_E4M3))
    return q, top[:, 0].contiguous()


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t, pad, op = _TYPES[case["dtype"]], case["pad"], case["op"]
    s = {"case": case}

    def vector(n, mid, scale):
        return (torch.randn(n, device="cuda", generator=g) * scale + mid).to(t)

    def f32(n):
        return torch.empty(n, dtype=torch.float32, device="cuda")

    if op in ("linear8", "gated8"):
        M, K, N = case["M"], case["K"], case["N" if op == "linear8" else "F"]
        s["x"], s["sx"] = _eight(g, M, K, pad, 1.0)
        if op == "linear8":
            s["w"], s["sw"] = _eight(g, N, K, pad, K ** -0.5)
            s["bias"] = vector(N, 0.0, 0.3) if case["bias"] else None
            s["res"] = _normal(g, M, N, pad, t, 1.0) if case["res"] else None
            s["y"] = _new(M, N, pad, t)
            s["z"] = _new(M, N, pad, t) if case["save"] else None
        else:
            s["wg"], s["sg"] = _eight(g, N, K, pad, K ** -0.5)
            s["wu"], s["su"] = _eight(g, N, K, pad, K ** -0.5)
            s["h"] = _new(M, N, pad, t)
            s["g"], s["u"] = (_new(M, N, pad, t), _new(M, N, pad, t)) if case["save"] else (None, None)
        return s
    r, c = case["rows"], case["cols"]
    if op.startswith("dropout"):
        s["x"] = _normal(g, r, c, pad, t, 1.0 if op == "dropout" else 0.1)
        s["r"] = _stream(g, r, c, pad, t) if case["res"] else None
        s["y"] = _new(r, c, pad, t)
        s["seed"], s["offset"] = 0x9E3779B97F4A7C15 ^ (seed * 0x1000193 + 1), 1000 + seed % 5000
        return s
    s["x"] = _stream(g, r, c, pad, t)
    if op == "rows8":
        s["q"], s["scale"] = _new(r, c, pad, _E4M3), f32(r)
        return s
    s["gamma"] = vector(c, 1.0, 0.2)
    if op == "rms_grad":
        s["rstd"] = (s["x"].double().square().mean(1) + _EPS).rsqrt().float()
        s["dy"] = _normal(g, r, c, pad, t, 0.1)
        s["ds"] = _normal(g, r, c, pad, t, 0.1) if case["res"] else None
        s["dx"], s["dgamma"] = _new(r, c, pad, t), f32(c)
        return s
    s["r"], s["s"] = (_normal(g, r, c, pad, t, 0.5), _new(r, c, pad, t)) if case["res"] else (None, None)
    if op == "rms":
        s["y"], s["rstd"] = _new(r, c, pad, t), f32(r)
    else:
        s["q"], s["scale"] = _new(r, c, pad, _E4M3), f32(r)
    return s


# ---- one pass -------------------------------------------------------------------------------------

def run(state):
    return (_run_own if own else _run_plain)(state, state["case"])


def _run_own(s, case):
    import paper_2003_00532_b200 as dg
    op = case["op"]
    if op == "rms":
        dg.rmsnorm_fwd(s["x"], s["gamma"], s["y"], eps=_EPS, residual=s["r"], sum=s["s"], rstd=s["rstd"])
        return {"y": s["y"], "s": s["s"], "rstd": s["rstd"]} if case["res"] else {"y": s["y"], "rstd": s["rstd"]}
    if op == "rms_grad":
        dg.rmsnorm_bwd(s["x"], s["gamma"], s["rstd"], s["dy"], dsum=s["ds"], dX=s["dx"], dgamma=s["dgamma"])
        return {"dx": s["dx"], "dgamma": s["dgamma"]}
    if op == "rms8":
        dg.rmsnorm_fwd_e4m3(s["x"], s["gamma"], s["q"], s["scale"], eps=_EPS, residual=s["r"], sum=s["s"])
        return {"q": s["q"], "scale": s["scale"], "s": s["s"]} if case["res"] else {"q": s["q"], "scale": s["scale"]}
    if op == "rows8":
        dg.quantize_rows_e4m3(s["x"], s["q"], s["scale"])
        return {"q": s["q"], "scale": s["scale"]}
    if op == "dropout":
        dg.dropout_fwd(s["x"], s["y"], case["p"], s["seed"], s["offset"], residual=s["r"])
        return {"y": s["y"]}
    if op == "dropout_grad":
        dg.dropout_bwd(s["x"], s["y"], case["p"], s["seed"], s["offset"])
        return {"dx": s["y"]}
    act = {"none": dg.HGEMM_ACT_NONE, "relu": dg.HGEMM_ACT_RELU, "gelu": dg.HGEMM_ACT_GELU,
           "gelu_tanh": dg.HGEMM_ACT_GELU_TANH, "silu": dg.HGEMM_ACT_SILU}[case["act"]]
    if op == "linear8":
        dg.qgemm_epilogue(s["x"], s["w"], s["y"], a_scale=s["sx"], b_scale=s["sw"], bias=s["bias"], act=act, residual=s["res"], preact=s["z"])
        return {"y": s["y"], "z": s["z"]} if case["save"] else {"y": s["y"]}
    dg.qgemm_gated(s["x"], s["wg"], s["wu"], s["h"], x_scale=s["sx"], g_scale=s["sg"], u_scale=s["su"], act=act, gate=s["g"], up=s["u"])
    return {"h": s["h"], "g": s["g"], "u": s["u"]} if case["save"] else {"h": s["h"]}


def _act(z, act):
    if act == "none":
        return z
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))
    return z / (1.0 + torch.exp(-z))


def _to_eight(y):
    """Rows of binary32 values as e4m3 with a scale each."""
    scale = y.abs().amax(1, keepdim=True).clamp_min(_LEAST) / _TOP
    return (y / scale).clamp(-_TOP, _TOP).to(_E4M3), scale[:, 0]


def _keep(rows, cols, p, seed, offset, device):
    """The mask of dropout: word c % 4 of Philox4x32-10 (Salmon et al., SC 2011) with the counter (c / 4, row, offset's halves) and the
    key seed, for column c, against p 2^32. 64-bit integers hold the 32-bit words; a product's high half is bits 32 to 63."""
    low = 0xFFFFFFFF
    a = torch.arange((cols + 3) // 4, dtype=torch.int64, device=device).expand(rows, -1)
    b = torch.arange(rows, dtype=torch.int64, device=device)[:, None].expand_as(a)
    c, d = torch.full_like(a, offset & low), torch.full_like(a, offset >> 32 & low)
    k0, k1 = seed & low, seed >> 32 & low
    for _ in range(10):
        x, y = a * 0xD2511F53, c * 0xCD9E8D57
        a, b, c, d = ((y >> 32) & low) ^ b ^ k0, y & low, ((x >> 32) & low) ^ d ^ k1, x & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    words = torch.stack((a, b, c, d), 2).reshape(rows, -1)[:, :cols]
    return words >= int(p * 2.0 ** 32 + 0.5)


def _run_plain(s, case):
    t, op = _TYPES[case["dtype"]], case["op"]
    x = s["x"].float()
    if op in ("rms", "rms8"):
        v = x + s["r"].float() if case["res"] else x
        rstd = torch.rsqrt((v * v).mean(1, keepdim=True) + _EPS)
        y = v * rstd * s["gamma"].float()
        out = {"s": v.to(t)} if case["res"] else {}
        if op == "rms":
            return dict(out, y=y.to(t), rstd=rstd[:, 0])
        q, scale = _to_eight(y)
        return dict(out, q=q, scale=scale)
    if op == "rms_grad":
        dy, rstd = s["dy"].float(), s["rstd"][:, None]
        xh = x * rstd
        w = dy * s["gamma"].float()
        dx = rstd * (w - xh * (w * xh).mean(1, keepdim=True))
        if case["res"]:
            dx = dx + s["ds"].float()
        return {"dx": dx.to(t), "dgamma": (dy * xh).sum(0)}
    if op == "rows8":
        q, scale = _to_eight(x)
        return {"q": q, "scale": scale}
    if op.startswith("dropout"):
        keep = _keep(case["rows"], case["cols"], case["p"], s["seed"], s["offset"], x.device)
        y = torch.where(keep, x * (1.0 / (1.0 - case["p"])), torch.zeros_like(x))
        if case["res"]:
            y = y + s["r"].float()
        return {"y" if op == "dropout" else "dx": y.to(t)}
    x = x * s["sx"][:, None]
    if op == "linear8":
        z = x @ (s["w"].float() * s["sw"][:, None]).t()
        if case["bias"]:
            z = z + s["bias"].float()
        y = _act(z, case["act"])
        if case["res"]:
            y = y + s["res"].float()
        return {"y": y.to(t), "z": z.to(t)} if case["save"] else {"y": y.to(t)}
    g, u = x @ (s["wg"].float() * s["sg"][:, None]).t(), x @ (s["wu"].float() * s["su"][:, None]).t()
    h = _act(g, case["act"]) * u
    return {"h": h.to(t), "g": g.to(t), "u": u.to(t)} if case["save"] else {"h": h.to(t)}


# ---- the definition in 64 bits ----------------------------------------------------------------------

def _nearest_e4m3(v):
    """The nearest e4m3 values: steps of 2^(e - 3) for values of exponent e, at least -6; ties to even."""
    step = torch.exp2(torch.frexp(v)[1].clamp_min(-5).double() - 4)
    return torch.round(v / step) * step


def _eight_exact(y):
    scale = torch.maximum(y.abs().max(1).values, torch.tensor(_LEAST, dtype=y.dtype, device=y.device)) / _TOP
    return _nearest_e4m3(y / scale[:, None]), scale


def _mask_exact(case, seed, offset):
    """The same generator in numpy's unsigned integers."""
    rows, cols = case["rows"], case["cols"]
    row, block = (a.ravel() for a in np.mgrid[0:rows, 0:-(-cols // 4)].astype(np.uint64))
    half, word = np.uint64(32), np.uint64(0xFFFFFFFF)
    w = [block, row, np.uint64(offset & 0xFFFFFFFF), np.uint64((offset >> 32) & 0xFFFFFFFF)]
    for i in range(10):
        key = [np.uint64(((seed >> 32 * j) + i * step) & 0xFFFFFFFF) for j, step in enumerate((0x9E3779B9, 0xBB67AE85))]
        p, q = w[0] * np.uint64(0xD2511F53), w[2] * np.uint64(0xCD9E8D57)
        w = [(q >> half) ^ w[1] ^ key[0], q & word, (p >> half) ^ w[3] ^ key[1], p & word]
    words = np.stack(np.broadcast_arrays(*w), axis=1).reshape(rows, -1)[:, :cols]
    return words.astype(np.float64) / 2.0 ** 32 >= round(case["p"] * 2 ** 32) / 2.0 ** 32


def _phi(z, act):
    if act == "none":
        return z
    if act == "relu":
        return z.clamp_min(0)
    if act == "silu":
        return z * torch.sigmoid(z)
    if act == "gelu":
        return z * torch.special.ndtr(z)
    return z * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    d = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor)}
    if op in ("rms", "rms8"):
        v = torch.add(d["x"], d["r"]) if case["res"] else d["x"]
        rstd = 1 / (torch.linalg.vector_norm(v, dim=1) ** 2 / case["cols"] + _EPS).sqrt()
        y = torch.einsum("rc,r,c->rc", v, rstd, d["gamma"])
        out = {"s": v} if case["res"] else {}
        if op == "rms":
            return {**out, "y": y, "rstd": rstd}
        q, scale = _eight_exact(y)
        return {**out, "q": q, "scale": scale}
    if op == "rms_grad":
        n, r = case["cols"], d["rstd"][:, None]
        w = d["dy"] * d["gamma"]
        # d/ds of s (s s / n + eps)^(-1/2): r w - r^3 s (s w) / n
        dx = r * w - r ** 3 / n * d["x"] * torch.einsum("rc,rc->r", d["x"], w)[:, None]
        if case["res"]:
            dx += d["ds"]
        return {"dx": dx, "dgamma": torch.einsum("rc,rc,r->c", d["dy"], d["x"], d["rstd"])}
    if op == "rows8":
        q, scale = _eight_exact(d["x"])
        return {"q": q, "scale": scale}
    if op.startswith("dropout"):
        mask = torch.from_numpy(_mask_exact(case, s["seed"], s["offset"])).to(d["x"].device)
        y = d["x"] * mask / (1 - case["p"])
        return {"y" if op == "dropout" else "dx": y + d["r"] if case["res"] else y}
    scaled = {k: torch.einsum("rk,r->rk", d[k], d[v]) for k, v in (("x", "sx"), ("w", "sw"), ("wg", "sg"), ("wu", "su")) if k in d}
    if op == "linear8":
        z = torch.einsum("mk,nk->mn", scaled["x"], scaled["w"])
        if case["bias"]:
            z += d["bias"]
        y = _phi(z, case["act"])
        if case["res"]:
            y = y + d["res"]
        return {"y": y, "z": z} if case["save"] else {"y": y}
    g, u = torch.einsum("mk,fk->mf", scaled["x"], scaled["wg"]), torch.einsum("mk,fk->mf", scaled["x"], scaled["wu"])
    h = _phi(g, case["act"]) * u
    return {"h": h, "g": g, "u": u} if case["save"] else {"h": h}
