"""A transformer's feed-forward sublayer on the library's 16-bit operators, forward and backward.

    y = x + (act(n Wg^T) * (n Wu^T)) Wd^T + bd,   n = layer norm of x

The normalisation, the gated projections and the product with bias and residual each run as one kernel
(:func:`layernorm_fwd`, :func:`hgemm_gated`, :func:`hgemm_epilogue`); the backward pass uses their gradients.
What lies between them is kept in the object's buffers, one per name, grown to the largest number of tokens so far; results are
new tensors. Run as a command it trains the sublayer on a synthetic target and then answers single tokens:

    python -m paper_2003_00532_b200.feed_forward [--model 1024] [--hidden 4096] [--tokens 2048] [--steps 20]
"""
from __future__ import annotations

import argparse
import time

import torch

import paper_2003_00532_b200 as dg


class FeedForward:
    """Weights of one sublayer (``float16`` or ``bfloat16``, stored output x input) and its two passes."""

    def __init__(self, model: int, hidden: int, dtype=torch.bfloat16, act: int = dg.HGEMM_ACT_SILU, seed: int = 0):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def weight(rows, cols):
            return (torch.randn(rows, cols, device="cuda", generator=g) * cols ** -0.5).to(dtype)

        self.model, self.hidden, self.dtype, self.act = model, hidden, dtype, act
        self.gamma, self.beta = torch.ones(model, dtype=dtype, device="cuda"), torch.zeros(model, dtype=dtype, device="cuda")
        self.wg, self.wu, self.wd = weight(hidden, model), weight(hidden, model), weight(model, hidden)
        self.bd = torch.zeros(model, dtype=dtype, device="cuda")
        self._buffers = {}
        self._kept = None

    def _buffer(self, name, tokens, *width, dtype=None):
        """``tokens`` rows of the buffer ``name``, which grows to the most tokens asked for and never shrinks."""
        if name not in self._buffers or self._buffers[name].shape[0] < tokens:
            self._buffers[name] = torch.empty(tokens, *width, dtype=dtype or self.dtype, device="cuda")
        return self._buffers[name][:tokens]

    def forward(self, x, keep: bool = True):
        """The sublayer's output for ``x`` (tokens x model), a new tensor. ``keep``: also keep what :meth:`backward` needs
        (``x`` itself by reference: it has to stay as it is until then); a call that does not keep leaves alone what an earlier
        one kept."""
        t, which = x.shape[0], "kept " if keep else ""
        n, h, y = self._buffer(which + "n", t, self.model), self._buffer(which + "h", t, self.hidden), torch.empty_like(x)
        mean, rstd, gate, up = None, None, None, None
        if keep:
            self._kept = None   # (its buffers are about to be written)
            mean, rstd = (self._buffer(name, t, dtype=torch.float32) for name in ("mean", "rstd"))
            gate, up = self._buffer("gate", t, self.hidden), self._buffer("up", t, self.hidden)
        dg.layernorm_fwd(x, self.gamma, self.beta, n, mean=mean, rstd=rstd)
        dg.hgemm_gated(n, self.wg, self.wu, h, act=self.act, gate=gate, up=up, transw=True)
        dg.hgemm_epilogue(h, self.wd, y, bias=self.bd, residual=x, transb=True)
        if keep:
            self._kept = (x, n, mean, rstd, gate, up, h)
        return y

    def backward(self, dy):
        """Gradients of the last kept :meth:`forward` for the incoming ``dy``: a dict of new tensors with ``x`` and every
        parameter's name."""
        if self._kept is None:
            raise RuntimeError("backward: no forward pass has been kept (forward(x, keep=True) comes first)")
        x, n, mean, rstd, gate, up, h = self._kept
        out = {name: torch.empty_like(getattr(self, name)) for name in ("wg", "wu", "wd")}
        out.update({name: torch.empty(self.model, dtype=torch.float32, device="cuda") for name in ("gamma", "beta", "bd")})
        t = x.shape[0]
        dh, dn, dx = self._buffer("dh", t, self.hidden), self._buffer("dn", t, self.model), torch.empty_like(x)
        dg.hgemm_epilogue_bwd(h, self.wd, dy, dA=dh, dB=out["wd"], dbias=out["bd"], transb=True)
        dg.hgemm_gated_bwd(n, self.wg, self.wu, gate, up, dh, act=self.act, dX=dn, dWg=out["wg"], dWu=out["wu"], transw=True)
        dg.layernorm_bwd(x, self.gamma, mean, rstd, dn, dX=dx, dgamma=out["gamma"], dbeta=out["beta"])
        out["x"] = dx.add_(dy)   # the residual
        return out

    def step(self, x, target, rate: float) -> float:
        """One step of gradient descent on the squared error per token (its sum over the model's width, averaged over the
        tokens); returns the mean squared error per value before it."""
        y = self.forward(x)
        diff = y.float() - target.float()
        grads = self.backward((diff * (2.0 / diff.shape[0])).to(self.dtype))
        for name in ("gamma", "beta", "wg", "wu", "wd", "bd"):
            p = getattr(self, name)
            p.copy_(p.float() - rate * grads[name].float())
        return float((diff * diff).mean())


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--model", type=int, default=1024)
    ap.add_argument("--hidden", type=int, default=4096)
    ap.add_argument("--tokens", type=int, default=2048)
    ap.add_argument("--steps", type=int, default=20)
    a = ap.parse_args()
    layer, teacher = FeedForward(a.model, a.hidden, seed=1), FeedForward(a.model, a.hidden, seed=2)
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
    torch.cuda.synchronize()
    t = time.perf_counter()
    for _ in range(200):
        layer.forward(x[:1], keep=False)
    torch.cuda.synchronize()
    print("answering: %.1f us per token, largest difference from the batch %.3g" % ((time.perf_counter() - t) / 200 * 1e6, off))


if __name__ == "__main__":
    main()
