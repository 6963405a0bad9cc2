"""The operators of a transformer's feed-forward path, as cases that can be measured: the 16-bit
matrix product with bias, activation and residual in its epilogue, the gated feed-forward
projections, and layer norm, each forward and backward.

``listed`` names fixed cases, ``draw`` makes more of the same ranges. ``prepare`` makes what a
program has in hand before a call (activations, weights, saved tensors, output buffers), ``run``
makes one pass: with ``own`` false in elementary 32-bit torch operations, with ``own`` true through
``paper_2003_00532_b200``. ``exact`` computes the same outputs in 64 bits. Matrices are row-major;
``pad`` elements are added to every leading dimension, as in the library's padded configurations.
"""
import math

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_BYTES = {"bf16": 2, "f16": 2, "f32": 4}
_EPS = 1e-5


def listed():
    return [
        # Output projection of one new token: 4096 x 4096 weights stored N x K, bias and residual. Latency
        # of the smallest product, bound by reading the weights.
        _linear("linear_token", "bf16", 1, 4096, 4096, act="none", bias=True, res=True, save=False, transb=True),
        # The library's ragged configuration (odd sizes, leading dimensions with odd padding) as a training
        # step's forward pass: weights stored K x N, everything in the epilogue, pre-activation kept.
        _linear("linear_ragged", "f16", 1000, 1537, 777, act="gelu", bias=True, res=True, save=True, transb=False, pad=3),
        # A long prompt or a training batch: compute-bound, the largest product.
        _linear("linear_batch", "bf16", 8192, 4096, 8192, act="gelu_tanh", bias=True, res=False, save=True, transb=True),
        # The gradients of such a layer at the library's 2088-row configuration: input, weight, bias.
        _linear("linear_grad", "bf16", 2088, 4096, 2088, act="gelu_tanh", bias=True, save=True, transb=True, back=True),
        # Gate and up projections of one new token of four requests: twice 4096 x 8192 weights to read.
        _gated("gated_tokens", "bf16", 4, 8192, 4096, act="silu", save=False, trans=True),
        # A ragged training batch in half precision: odd row count, both pre-activations kept.
        _gated("gated_batch", "f16", 4097, 8192, 2048, act="silu", save=True, trans=True),
        # The backward pass of the gated projections: input gradient and both weight gradients.
        _gated("gated_grad", "bf16", 4096, 8192, 2048, act="silu", save=True, trans=True, back=True),
        # A short ragged batch's gradients, weights stored K x F: too few tiles to fill the GPU.
        _gated("gated_grad_short", "bf16", 333, 1537, 1000, act="gelu_tanh", save=True, trans=False, back=True),
        # Layer norm of one new token: the smallest call of all, latency alone.
        _norm("norm_token", "bf16", 1, 4096),
        # Layer norm of a training batch, with the row statistics kept: bound by memory.
        _norm("norm_batch", "bf16", 8192, 4096),
        # Its backward pass with the reduction of both parameter gradients over the rows.
        _norm("norm_grad", "bf16", 8192, 4096, back=True),
        # The same in single precision on the ragged row length, rows that are not 16-byte aligned.
        _norm("norm_grad_ragged", "f32", 4097, 1537, pad=3, back=True),
    ]


def _linear(name, dtype, M, N, K, *, act, bias, save, transb, res=False, pad=0, back=False):
    c = {"op": "linear_grad" if back else "linear", "dtype": dtype, "M": M, "N": N, "K": K, "act": act, "bias": bias,
         "res": res, "save": save, "trans": transb, "pad": pad}
    return dict(c, name=name) if name else c


def _gated(name, dtype, M, F, K, *, act, save, trans, pad=0, back=False):
    c = {"op": "gated_grad" if back else "gated", "dtype": dtype, "M": M, "F": F, "K": K, "act": act, "save": save,
         "trans": trans, "pad": pad}
    return dict(c, name=name) if name else c


def _norm(name, dtype, rows, cols, *, pad=0, back=False):
    c = {"op": "norm_grad" if back else "norm", "dtype": dtype, "rows": rows, "cols": cols, "pad": pad}
    return dict(c, name=name) if name else c


def _size(rng, lo, hi):
    """Log-uniform in lo..hi; every other one brought to a multiple of 64 or 8, the rest as they fall."""
    n = math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))
    step = rng.choice([1, 1, 8, 64])
    return min(hi, max(lo, int(round(n / step)) * step))


def draw(rng):
    op = rng.choice(["linear", "linear", "linear_grad", "gated", "gated", "gated_grad", "norm", "norm_grad"])
    if op.startswith("norm"):
        while True:
            rows, cols = _size(rng, 1, 16384), _size(rng, 32, 16384)
            if rows * cols <= 8192 * 4096:
                break
        return _norm(None, rng.choice(["bf16", "f16", "f32"]), rows, cols, pad=rng.choice([0, 0, 8, 3]), back=op == "norm_grad")
    back = op.endswith("grad")
    dtype, trans, pad = rng.choice(["bf16", "f16"]), rng.random() < 0.5, rng.choice([0, 0, 0, 8, 3])
    while True:
        M, N, K = _size(rng, 1, 8192), _size(rng, 64, 8192), _size(rng, 64, 8192)
        flops = 2.0 * M * N * K * (2 if back else 1) * (2 if op.startswith("gated") else 1)
        if flops <= 2.0 * 8192 * 4096 * 8192:
            break
    if op.startswith("gated"):
        return _gated(None, dtype, M, N, K, act=rng.choice(["silu", "gelu_tanh", "gelu"]), save=back or rng.random() < 0.5, trans=trans, pad=pad, back=back)
    act = rng.choice(["none", "relu", "gelu", "gelu_tanh", "silu"])
    return _linear(None, dtype, M, N, K, act=act, bias=rng.random() < 0.7, save=(back or rng.random() < 0.5) and act != "none",
                   transb=trans, res=not back and rng.random() < 0.5, pad=pad, back=back)


def work(case):
    e = _BYTES[case["dtype"]]
    op = case["op"]
    if op.startswith("norm"):
        n, r, c = case["rows"] * case["cols"], case["rows"], case["cols"]
        if op == "norm":  # x, gamma, beta in; y, mean, rstd out
            return {"bytes": 2 * n * e + 2 * c * e + 8 * r, "flops": 8 * n}
        return {"bytes": 3 * n * e + c * e + 8 * r + 8 * c, "flops": 14 * n}  # x, dy, gamma, mean, rstd in; dx, dgamma, dbeta out
    if op.startswith("linear"):
        M, N, K = case["M"], case["N"], case["K"]
        if op == "linear":
            return {"bytes": e * (M * K + K * N + M * N * (1 + case["res"] + case["save"]) + N * case["bias"]), "flops": 2 * M * N * K}
        return {"bytes": e * (2 * (M * K + K * N) + M * N * (1 + case["save"])) + 4 * N * case["bias"], "flops": 4 * M * N * K}
    M, F, K = case["M"], case["F"], case["K"]
    if op == "gated":
        return {"bytes": e * (M * K + 2 * K * F + M * F * (3 if case["save"] else 1)), "flops": 4 * M * F * K}
    return {"bytes": e * (2 * M * K + 4 * K * F + 3 * M * F), "flops": 8 * M * F * K}


# ---- inputs ---------------------------------------------------------------------------------------

def _new(rows, cols, pad, t):
    return torch.empty(rows, cols + pad, dtype=t, device="cuda")[:, :cols]


def _normal(g, rows, cols, pad, t, scale):
    x = _new(rows, cols, pad, t)
    x.copy_(torch.randn(rows, cols, device="cuda", generator=g) * scale)
    return x


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t, pad, op = _TYPES[case["dtype"]], case["pad"], case["op"]
    s = {"case": case}

    def normal(rows, cols, scale):
        return _normal(g, rows, cols, pad, t, scale)

    def vector(n, mid, scale):
        return (torch.randn(n, device="cuda", generator=g) * scale + mid).to(t)

    def f32(n):
        return torch.empty(n, dtype=torch.float32, device="cuda")

    def weights(K, N):
        return normal(N, K, K ** -0.5) if case["trans"] else normal(K, N, K ** -0.5)

    if op.startswith("norm"):
        r, c = case["rows"], case["cols"]
        # the residual stream: rows of different size, a mean of their own
        s["x"] = _new(r, c, pad, t)
        s["x"].copy_(torch.randn(r, c, device="cuda", generator=g) * (0.5 + 2 * torch.rand(r, 1, device="cuda", generator=g))
                     + 0.3 * torch.randn(r, 1, device="cuda", generator=g))
        s["gamma"] = vector(c, 1.0, 0.2)
        if op == "norm":
            s["beta"] = vector(c, 0.0, 0.2)
            s["y"], s["mean"], s["rstd"] = _new(r, c, pad, t), f32(r), f32(r)
        else:
            x = s["x"].double()
            s["mean"] = x.mean(1).float()
            s["rstd"] = (x.var(1, unbiased=False) + _EPS).rsqrt().float()
            s["dy"] = normal(r, c, 0.1)
            s["dx"], s["dgamma"], s["dbeta"] = _new(r, c, pad, t), f32(c), f32(c)
        return s
    M, K = case["M"], case["K"]
    s["x"] = normal(M, K, 1.0)
    if op.startswith("linear"):
        N = case["N"]
        s["w"] = weights(K, N)
        s["bias"] = vector(N, 0.0, 0.3) if case["bias"] else None
        if op == "linear":
            s["res"] = normal(M, N, 1.0) if case["res"] else None
            s["y"] = _new(M, N, pad, t)
            s["z"] = _new(M, N, pad, t) if case["save"] else None
        else:
            s["z"] = None
            if case["save"]:
                s["z"] = _new(M, N, pad, t)
                s["z"].copy_(torch.matmul(s["x"], s["w"].t() if case["trans"] else s["w"]) + (s["bias"] if case["bias"] else 0))
            s["dy"] = normal(M, N, 0.1)
            s["dx"], s["dw"] = _new(M, K, pad, t), _new(*s["w"].shape, pad, t)
            s["db"] = f32(N) if case["bias"] else None
        return s
    F = case["F"]
    s["wg"], s["wu"] = weights(K, F), weights(K, F)
    if op == "gated":
        s["h"] = _new(M, F, pad, t)
        s["g"], s["u"] = (_new(M, F, pad, t), _new(M, F, pad, t)) if case["save"] else (None, None)
    else:
        s["g"], s["u"] = _new(M, F, pad, t), _new(M, F, pad, t)
        for name, w in (("g", s["wg"]), ("u", s["wu"])):
            s[name].copy_(torch.matmul(s["x"], w.t() if case["trans"] else w))
        s["dh"] = normal(M, F, 0.1)
        s["dx"], s["dwg"], s["dwu"] = _new(M, K, pad, t), _new(*s["wg"].shape, pad, t), _new(*s["wu"].shape, pad, t)
    return s


# ---- one pass -------------------------------------------------------------------------------------

def run(state):
    return (_run_own if own else _run_plain)(state, state["case"])


def _run_own(s, case):
    import paper_2003_00532_b200 as dg
    op = case["op"]
    if op == "norm":
        dg.layernorm_fwd(s["x"], s["gamma"], s["beta"], s["y"], eps=_EPS, mean=s["mean"], rstd=s["rstd"])
        return {"y": s["y"], "mean": s["mean"], "rstd": s["rstd"]}
    if op == "norm_grad":
        dg.layernorm_bwd(s["x"], s["gamma"], s["mean"], s["rstd"], s["dy"], dX=s["dx"], dgamma=s["dgamma"], dbeta=s["dbeta"])
        return {"dx": s["dx"], "dgamma": s["dgamma"], "dbeta": s["dbeta"]}
    act = {"none": dg.HGEMM_ACT_NONE, "relu": dg.HGEMM_ACT_RELU, "gelu": dg.HGEMM_ACT_GELU,
           "gelu_tanh": dg.HGEMM_ACT_GELU_TANH, "silu": dg.HGEMM_ACT_SILU}[case["act"]]
    if op == "linear":
        dg.hgemm_epilogue(s["x"], s["w"], s["y"], bias=s["bias"], act=act, residual=s["res"], preact=s["z"], transb=case["trans"])
        return {"y": s["y"], "z": s["z"]} if case["save"] else {"y": s["y"]}
    if op == "linear_grad":
        dg.hgemm_epilogue_bwd(s["x"], s["w"], s["dy"], act=act, preact=s["z"], dA=s["dx"], dB=s["dw"], dbias=s["db"], transb=case["trans"])
        return {"dx": s["dx"], "dw": s["dw"], "db": s["db"]} if case["bias"] else {"dx": s["dx"], "dw": s["dw"]}
    if op == "gated":
        dg.hgemm_gated(s["x"], s["wg"], s["wu"], s["h"], act=act, gate=s["g"], up=s["u"], transw=case["trans"])
        return {"h": s["h"], "g": s["g"], "u": s["u"]} if case["save"] else {"h": s["h"]}
    dg.hgemm_gated_bwd(s["x"], s["wg"], s["wu"], s["g"], s["u"], s["dh"], act=act, dX=s["dx"], dWg=s["dwg"], dWu=s["dwu"], transw=case["trans"])
    return {"dx": s["dx"], "dwg": s["dwg"], "dwu": s["dwu"]}


def _sigmoid(z):
    return 1.0 / (1.0 + torch.exp(-z))


def _act(z, act):
    if act == "none":
        return z
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))
    return z * _sigmoid(z)


def _act_grad(z, act):
    if act == "none":
        return torch.ones_like(z)
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    if act == "gelu_tanh":
        c = math.sqrt(2.0 / math.pi)
        t = torch.tanh(c * (z + 0.044715 * z * z * z))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * c * (1.0 + 3 * 0.044715 * z * z)
    q = _sigmoid(z)
    return q * (1.0 + z * (1.0 - q))


def _run_plain(s, case):
    t, op = _TYPES[case["dtype"]], case["op"]
    x = s["x"].float()
    if op == "norm":
        mean = x.mean(1, keepdim=True)
        d = x - mean
        rstd = torch.rsqrt((d * d).mean(1, keepdim=True) + _EPS)
        y = d * rstd * s["gamma"].float() + s["beta"].float()
        return {"y": y.to(t), "mean": mean[:, 0], "rstd": rstd[:, 0]}
    if op == "norm_grad":
        dy, rstd = s["dy"].float(), s["rstd"][:, None]
        xhat = (x - s["mean"][:, None]) * rstd
        w = dy * s["gamma"].float()
        dx = rstd * (w - w.mean(1, keepdim=True) - xhat * (w * xhat).mean(1, keepdim=True))
        return {"dx": dx.to(t), "dgamma": (dy * xhat).sum(0), "dbeta": dy.sum(0)}
    act, trans = case["act"], case["trans"]
    if op.startswith("linear"):
        w = s["w"].float()
        w = w.t() if trans else w
        if op == "linear":
            z = x @ w
            if case["bias"]:
                z = z + s["bias"].float()
            y = _act(z, act)
            if case["res"]:
                y = y + s["res"].float()
            return {"y": y.to(t), "z": z.to(t)} if case["save"] else {"y": y.to(t)}
        dz = s["dy"].float()
        if act != "none":
            dz = dz * _act_grad(s["z"].float(), act)
        dw = (dz.t() @ x) if trans else (x.t() @ dz)
        out = {"dx": (dz @ w.t()).to(t), "dw": dw.to(t)}
        if case["bias"]:
            out["db"] = dz.sum(0)
        return out
    wg, wu = s["wg"].float(), s["wu"].float()
    if trans:
        wg, wu = wg.t(), wu.t()
    if op == "gated":
        g, u = x @ wg, x @ wu
        h = _act(g, act) * u
        return {"h": h.to(t), "g": g.to(t), "u": u.to(t)} if case["save"] else {"h": h.to(t)}
    g, u, dh = s["g"].float(), s["u"].float(), s["dh"].float()
    dg = dh * u * _act_grad(g, act)
    du = dh * _act(g, act)
    dx = dg @ wg.t() + du @ wu.t()
    dwg, dwu = (dg.t() @ x, du.t() @ x) if trans else (x.t() @ dg, x.t() @ du)
    return {"dx": dx.to(t), "dwg": dwg.to(t), "dwu": dwu.to(t)}


# ---- the definition in 64 bits ----------------------------------------------------------------------

def _phi(z, act):
    """The activation and its derivative, in the type of z."""
    if act == "none":
        return z, z * 0 + 1
    if act == "relu":
        return z.clamp_min(0), torch.heaviside(z, torch.zeros((), dtype=z.dtype, device=z.device))
    if act == "silu":
        q = torch.sigmoid(z)
        return z * q, q + z * q * (1 - q)
    if act == "gelu":
        cdf = torch.special.ndtr(z)
        return z * cdf, cdf + z * (-(z ** 2) / 2).exp() / math.sqrt(2 * math.pi)
    # z sigmoid(2 p(z)) with p the cubic inside the tanh
    c = math.sqrt(2 / math.pi)
    q = torch.sigmoid(2 * c * (z + 0.044715 * z ** 3))
    return z * q, q + z * q * (1 - q) * 2 * c * (1 + 0.134145 * z ** 2)


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    d = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor)}
    if op == "norm":
        n = case["cols"]
        mean = d["x"].sum(1) / n
        var = ((d["x"] - mean[:, None]) ** 2).sum(1) / n
        rstd = 1 / (var + _EPS).sqrt()
        return {"y": torch.addcmul(d["beta"], (d["x"] - mean[:, None]) * rstd[:, None], d["gamma"]), "mean": mean, "rstd": rstd}
    if op == "norm_grad":
        n = case["cols"]
        xh = (d["x"] - d["mean"][:, None]) * d["rstd"][:, None]
        dxh = d["dy"] * d["gamma"]
        dx = d["rstd"][:, None] / n * (n * dxh - dxh.sum(1, keepdim=True) - xh * (dxh * xh).sum(1, keepdim=True))
        return {"dx": dx, "dgamma": torch.einsum("rc,rc->c", d["dy"], xh), "dbeta": d["dy"].sum(0)}
    form = "mk,nk->mn" if case["trans"] else "mk,kn->mn"
    if op == "linear":
        z = torch.einsum(form, d["x"], d["w"])
        if case["bias"]:
            z += d["bias"]
        y = _phi(z, case["act"])[0]
        if case["res"]:
            y = y + d["res"]
        return {"y": y, "z": z} if case["save"] else {"y": y}
    to_x = "mn,nk->mk" if case["trans"] else "mn,kn->mk"
    to_w = "mn,mk->nk" if case["trans"] else "mn,mk->kn"
    if op == "linear_grad":
        dz = d["dy"] if case["act"] == "none" else d["dy"] * _phi(d["z"], case["act"])[1]
        out = {"dx": torch.einsum(to_x, dz, d["w"]), "dw": torch.einsum(to_w, dz, d["x"])}
        if case["bias"]:
            out["db"] = dz.sum(0)
        return out
    if op == "gated":
        g, u = torch.einsum(form, d["x"], d["wg"]), torch.einsum(form, d["x"], d["wu"])
        h = _phi(g, case["act"])[0] * u
        return {"h": h, "g": g, "u": u} if case["save"] else {"h": h}
    a, da = _phi(d["g"], case["act"])
    dg, du = d["dh"] * d["u"] * da, d["dh"] * a
    dx = torch.einsum(to_x, dg, d["wg"]) + torch.einsum(to_x, du, d["wu"])
    return {"dx": dx, "dwg": torch.einsum(to_w, dg, d["x"]), "dwu": torch.einsum(to_w, du, d["x"])}
