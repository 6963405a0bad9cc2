"""A transformer's feed-forward sublayer on the library's 16-bit operators, forward and backward, and on its 8-bit operators for
answering.

    s = x + delta,   y = s + dropout((act(n Wg^T) * (n Wu^T)) Wd^T + bd),   n = norm of s

The norm is layer norm or root-mean-square norm; ``delta`` is what the sublayer before leaves to be added to the residual stream
(root-mean-square norm adds it in its own pass). The normalisation, the gated projections and the product with bias and residual each
run as one kernel (:func:`layernorm_fwd` or :func:`rmsnorm_fwd`, :func:`hgemm_gated`, :func:`hgemm_epilogue`, and :func:`dropout_fwd`
behind it); the backward pass uses their gradients. What lies between them is kept in the object's buffers, one per name, grown to the
largest number of tokens so far; results are new tensors. :meth:`FeedForward.eight_bit` gives the sublayer with its weights in 8 bits,
whose activations are brought there by :func:`rmsnorm_fwd_e4m3` and :func:`quantize_rows_e4m3` and multiplied by
:func:`qgemm_gated` and :func:`qgemm_epilogue`. Run as a command it trains the sublayer on a synthetic target and then answers
single tokens:

    python -m paper_2003_00532_b200.feed_forward [--model 1024] [--hidden 4096] [--tokens 2048] [--steps 20] [--norm rms] [--dropout 0.1]
"""
from __future__ import annotations

import argparse
import time

import torch

import paper_2003_00532_b200 as dg


class _Buffers:
    """Scratch tensors by name, each grown to the most tokens asked for. One that a captured pass was given stays for the object's life,
    also when a larger one takes its place: the graph writes to it in every replay.

    The next pass writes over them: an object's passes, replays among them, follow one another on one stream or are made to wait for each
    other, and belong to one thread at a time."""

    def __init__(self):
        self._buffers, self._captured, self._capturing = {}, [], False

    def _begin(self):
        """Called once at the beginning of a pass (asked of CUDA for every buffer, a token's pass took 1 to 2 us longer)."""
        self._capturing = torch.cuda.is_current_stream_capturing()

    def _buffer(self, name, tokens, *width, dtype=None):
        """``tokens`` rows of the buffer ``name``, which grows to the most tokens asked for and never shrinks."""
        buffer = self._buffers.get(name)
        if buffer is None or buffer.shape[0] < tokens:
            buffer = self._buffers[name] = torch.empty(tokens, *width, dtype=dtype or self.dtype, device="cuda")
        if self._capturing and not any(held is buffer for held in self._captured):
            self._captured.append(buffer)
        return buffer[:tokens]


#: Where the masks of captured passes begin among the uses of a seed; those of other passes begin at 0.
CAPTURED_USES = 1 << 62


class FeedForward(_Buffers):
    """Weights of one sublayer (``float16`` or ``bfloat16``, stored output x input) and its two passes. ``norm``: ``"layer"`` or
    ``"rms"``; ``dropout``: the probability with which a kept (training) pass drops a value of the sublayer's output."""

    def __init__(self, model: int, hidden: int, dtype=torch.bfloat16, act: int = dg.HGEMM_ACT_SILU, seed: int = 0, norm: str = "layer",
                 dropout: float = 0.0):
        super().__init__()
        if norm not in ("layer", "rms"):
            raise ValueError("norm: 'layer' or 'rms'")
        if not 0.0 <= dropout < 1.0:
            raise ValueError("dropout: a probability below 1")
        g = torch.Generator(device="cuda").manual_seed(seed)

        def weight(rows, cols):
            return (torch.randn(rows, cols, device="cuda", generator=g) * cols ** -0.5).to(dtype)

        self.model, self.hidden, self.dtype, self.act = model, hidden, dtype, act
        self.norm, self.dropout, self.seed, self.uses = norm, dropout, seed, 0
        self._replays = torch.zeros(1, dtype=torch.int64, device="cuda")   # passes of captured graphs, counted when they run
        self.gamma = torch.ones(model, dtype=dtype, device="cuda")
        self.beta = torch.zeros(model, dtype=dtype, device="cuda") if norm == "layer" else None
        self.wg, self.wu, self.wd = weight(hidden, model), weight(hidden, model), weight(model, hidden)
        self.bd = torch.zeros(model, dtype=dtype, device="cuda")
        self._kept = None

    def parameters(self):
        """The parameters' names."""
        return ("gamma", "beta", "wg", "wu", "wd", "bd") if self.norm == "layer" else ("gamma", "wg", "wu", "wd", "bd")

    def forward(self, x, keep: bool = True, delta=None):
        """The sublayer's output for ``x`` (tokens x model), a new tensor. ``keep``: also keep what :meth:`backward` needs
        (``x`` itself by reference: it has to stay as it is until then) and drop values, with another mask every time, also in every
        replay of a captured call (whose gradients are taken before the next replay); a call that does not keep drops nothing and leaves
        alone what an earlier one kept. ``delta`` (root-mean-square norm only): added to ``x`` first."""
        if delta is not None and self.norm != "rms":
            raise ValueError("delta: needs norm='rms'")
        self._begin()
        t, which = x.shape[0], "kept " if keep else ""
        n, h, y = self._buffer(which + "n", t, self.model), self._buffer(which + "h", t, self.hidden), torch.empty_like(x)
        mean, rstd, gate, up = None, None, None, None
        if keep:
            self._kept = None   # (its buffers are about to be written)
            mean, rstd = (self._buffer(name, t, dtype=torch.float32) for name in ("mean", "rstd"))
            gate, up = self._buffer("gate", t, self.hidden), self._buffer("up", t, self.hidden)
        s = x
        if self.norm == "layer":
            dg.layernorm_fwd(x, self.gamma, self.beta, n, mean=mean, rstd=rstd)
        else:
            if delta is not None:
                s = self._buffer(which + "s", t, self.model)
            dg.rmsnorm_fwd(x, self.gamma, n, residual=delta, sum=s if delta is not None else None, rstd=rstd)
        dg.hgemm_gated(n, self.wg, self.wu, h, act=self.act, gate=gate, up=up, transw=True)
        p, use, step = self.dropout if keep else 0.0, self.uses, None
        if p > 0.0:
            if self._capturing:
                use, step = CAPTURED_USES, self._replays.add_(1)
            else:
                self.uses += 1
            d = self._buffer("d", t, self.model)
            dg.hgemm_epilogue(h, self.wd, d, bias=self.bd, transb=True)
            dg.dropout_fwd(d, y, p, self.seed, use, residual=s, step=step)
        else:
            dg.hgemm_epilogue(h, self.wd, y, bias=self.bd, residual=s, transb=True)
        if keep:
            self._kept = (s, n, mean, rstd, gate, up, h, p, use, step)
        return y

    def backward(self, dy):
        """Gradients of the last kept :meth:`forward` for the incoming ``dy``: a dict of new tensors with ``x`` (which is ``delta``'s,
        too) and every parameter's name."""
        if self._kept is None:
            raise RuntimeError("backward: no forward pass has been kept (forward(x, keep=True) comes first)")
        self._begin()
        s, n, mean, rstd, gate, up, h, p, use, step = self._kept
        out = {name: torch.empty_like(getattr(self, name)) for name in ("wg", "wu", "wd")}
        out.update({name: torch.empty(self.model, dtype=torch.float32, device="cuda") for name in self.parameters() if name not in out})
        t = s.shape[0]
        dh, dn, dx = self._buffer("dh", t, self.hidden), self._buffer("dn", t, self.model), torch.empty_like(s)
        dd = dy
        if p > 0.0:
            dd = self._buffer("d", t, self.model)
            dg.dropout_bwd(dy, dd, p, self.seed, use, step=step)
        dg.hgemm_epilogue_bwd(h, self.wd, dd, dA=dh, dB=out["wd"], dbias=out["bd"], transb=True)
        dg.hgemm_gated_bwd(n, self.wg, self.wu, gate, up, dh, act=self.act, dX=dn, dWg=out["wg"], dWu=out["wu"], transw=True)
        if self.norm == "layer":
            dg.layernorm_bwd(s, self.gamma, mean, rstd, dn, dX=dx, dgamma=out["gamma"], dbeta=out["beta"])
            out["x"] = dx.add_(dy)   # the residual
        else:
            dg.rmsnorm_bwd(s, self.gamma, rstd, dn, dsum=dy, dX=dx, dgamma=out["gamma"])   # the residual's gradient joins
            out["x"] = dx
        return out

    def eight_bit(self):
        """The sublayer for answering, its weights in 8 bits with a scale per row (root-mean-square norm only)."""
        return EightBitFeedForward(self)

    def step(self, x, target, rate: float) -> float:
        """One step of gradient descent on the squared error per token (its sum over the model's width, averaged over the
        tokens); returns the mean squared error per value before it."""
        y = self.forward(x)
        diff = y.float() - target.float()
        grads = self.backward((diff * (2.0 / diff.shape[0])).to(self.dtype))
        for name in self.parameters():
            p = getattr(self, name)
            p.copy_(p.float() - rate * grads[name].float())
        return float((diff * diff).mean())


class EightBitFeedForward(_Buffers):
    """A sublayer's forward pass with weights and activations in 8 bits (e4m3), a scale for each weight row and token."""

    def __init__(self, layer: FeedForward):
        super().__init__()
        if layer.norm != "rms":
            raise ValueError("eight_bit: needs norm='rms'")
        self.model, self.hidden, self.dtype, self.act = layer.model, layer.hidden, layer.dtype, layer.act
        self.gamma, self.bd = layer.gamma.clone(), layer.bd.clone()
        for name in ("wg", "wu", "wd"):
            w = getattr(layer, name)
            q = torch.empty(w.shape, dtype=torch.float8_e4m3fn, device="cuda")
            scale = torch.empty(w.shape[0], dtype=torch.float32, device="cuda")
            dg.quantize_rows_e4m3(w, q, scale)
            setattr(self, name, q)
            setattr(self, "s" + name[1:], scale)

    def forward(self, x, delta=None):
        """As :meth:`FeedForward.forward` with ``keep=False``."""
        self._begin()
        t, e4m3, f32 = x.shape[0], torch.float8_e4m3fn, torch.float32
        n, sn = self._buffer("n", t, self.model, dtype=e4m3), self._buffer("sn", t, dtype=f32)
        h, y = self._buffer("h", t, self.hidden), torch.empty_like(x)
        q, sq = self._buffer("q", t, self.hidden, dtype=e4m3), self._buffer("sq", t, dtype=f32)
        s = x if delta is None else self._buffer("s", t, self.model)
        dg.rmsnorm_fwd_e4m3(x, self.gamma, n, sn, residual=delta, sum=None if delta is None else s)
        dg.qgemm_gated(n, self.wg, self.wu, h, x_scale=sn, g_scale=self.sg, u_scale=self.su, act=self.act)
        dg.quantize_rows_e4m3(h, q, sq)
        dg.qgemm_epilogue(q, self.wd, y, a_scale=sq, b_scale=self.sd, bias=self.bd, residual=s)
        return y


def _time_per_token(layer, x, **more) -> float:
    """Microseconds of one token's pass."""
    layer.forward(x[:1], **more)
    torch.cuda.synchronize()
    t = time.perf_counter()
    for _ in range(200):
        layer.forward(x[:1], **more)
    torch.cuda.synchronize()
    return (time.perf_counter() - t) / 200 * 1e6


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--model", type=int, default=1024)
    ap.add_argument("--hidden", type=int, default=4096)
    ap.add_argument("--tokens", type=int, default=2048)
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--norm", choices=("layer", "rms"), default="layer")
    ap.add_argument("--dropout", type=float, default=0.0)
    a = ap.parse_args()
    layer, teacher = FeedForward(a.model, a.hidden, seed=1, norm=a.norm, dropout=a.dropout), FeedForward(a.model, a.hidden, seed=2, norm=a.norm)
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(a.tokens, a.model, device="cuda", generator=g).to(layer.dtype)
    target = teacher.forward(x, keep=False)
    losses = [layer.step(x, target, 0.05) for _ in range(a.steps)]
    status = dg.hgemm_last_device_status()
    if status != dg.DGEMM_OK:
        raise dg.DgemmError(status, "feed_forward")
    print("training: loss %.4f -> %.4f in %d steps of %d tokens" % (losses[0], losses[-1], a.steps, a.tokens))
    # answering: one token at a time gives what the whole batch gives, up to the rounding of 16 bits
    batch = layer.forward(x[:8], keep=False)
    rows = [layer.forward(x[i:i + 1], keep=False) for i in range(8)]
    off = float((torch.cat(rows).float() - batch.float()).abs().max())
    print("answering: %.1f us per token, largest difference from the batch %.3g" % (_time_per_token(layer, x, keep=False), off))
    if a.norm == "rms":
        eight = layer.eight_bit()
        far = float((eight.forward(x[:8]).float() - batch.float()).norm() / (batch.float() - x[:8].float()).norm())
        print("answering in 8 bits: %.1f us per token, off by %.3g of the sublayer's part" % (_time_per_token(eight, x), far))


if __name__ == "__main__":
    main()
