"""The feed-forward sublayer with root-mean-square norm, the residual's addition and dropout, forward and backward, against the same
sublayer in 64 bits with torch's own differentiation; and its form in 8 bits. Needs a B200.

Tolerance of the 16-bit sublayer: at most nine roundings to 16 bits lie on any path from an input to an output or gradient (the sum, n,
gate, up, h, the product before dropout, what dropout leaves of dy, dh, dn or the result itself), each off by u of the value with
independent signs: relative error of a whole matrix (2-norm) below 9 u.

Tolerance of the 8-bit sublayer against its own definition (weights as they were brought to 8 bits, activations brought there in 64 bits):
the 64-bit values before a rounding to e4m3 agree with the kernels' to 2^-15 (norm) or to the rounding of h to 16 bits, so that a share
of the values, at most 2 e / step for a difference of e, falls to the other neighbour, a step of 2^-3 away: the error they leave has a mean
square of at most e step. For n: e = 2^-14 relative, step 2^-3: 2^-17, a relative error below 2^-8 in gate, up and h. For h: e = 2^-8 +
u, step 2^-3: below 2^-10 in the mean square, 2^-5 relative, which the product passes on."""
import pytest
import torch

import hgemm_reference as ref
import paper_2003_00532_b200 as dg
import rows_reference as rr
from paper_2003_00532_b200.feed_forward import FeedForward

pytestmark = pytest.mark.gpu

U = ref.U


def _exact(layer, x, delta, keep=None):
    names = layer.parameters()
    p = {k: getattr(layer, k).double().requires_grad_() for k in names}
    p["x"] = x.double().requires_grad_()
    s = p["x"] if delta is None else p["x"] + delta.double()
    n = s * (s.square().mean(1, keepdim=True) + 1e-5).rsqrt() * p["gamma"]
    g = n @ p["wg"].t()
    f = (g * torch.sigmoid(g) * (n @ p["wu"].t())) @ p["wd"].t() + p["bd"]
    return p, s + (f if keep is None else f * keep / (1 - layer.dropout))


def _layer(model, hidden, dtype, seed, **more):
    layer = FeedForward(model, hidden, dtype=dtype, seed=seed, norm="rms", **more)
    g = torch.Generator(device="cuda").manual_seed(5)
    layer.gamma.add_(torch.randn(model, device="cuda", generator=g) * 0.2)
    layer.bd.add_(torch.randn(model, device="cuda", generator=g) * 0.2)
    return layer, g


def _close(a, b, dtype, what, most=None):
    rel = float((a.double() - b).norm() / b.norm())
    assert rel <= (most or 9 * U[dtype]), f"{what}: {rel:.3g}"


SIZES = [(1, 64, 100), (2, 256, 512), (37, 200, 333), (300, 520, 1000), (1024, 1024, 2048)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("dropout", [0.0, 0.2])
@pytest.mark.parametrize("tokens,model,hidden", SIZES)
def test_sublayer_and_gradients(tokens, model, hidden, dropout, dtype):
    layer, g = _layer(model, hidden, dtype, tokens, dropout=dropout)
    x, delta, dy = (torch.randn(tokens, model, device="cuda", generator=g).to(dtype) for _ in range(3))
    for use in range(2):               # a second pass drops others
        y = layer.forward(x, delta=delta)
        got = layer.backward(dy)
        assert dg.hgemm_last_device_status() == dg.DGEMM_OK
        keep = rr.words(tokens, model, layer.seed, use, "cuda") >= int(dropout * 2 ** 32 + 0.5) if dropout else None
        p, want = _exact(layer, x, delta, keep)
        want.backward(dy.double())
        _close(y, want.detach(), dtype, "y")
        for k in got:
            _close(got[k], p[k].grad, dtype, k)
    _close(layer.forward(x, keep=False, delta=delta), _exact(layer, x, delta)[1].detach(), dtype, "without dropout")


def test_without_an_addition_and_tokens_agree_with_the_batch():
    layer, g = _layer(256, 512, torch.bfloat16, 1)
    x = torch.randn(6, 256, device="cuda", generator=g).bfloat16()
    batch = layer.forward(x, keep=False)
    _close(batch, _exact(layer, x, None)[1].detach(), torch.bfloat16, "batch")
    rows = torch.cat([layer.forward(x[i:i + 1], keep=False) for i in range(6)])
    _close(rows, batch.double(), torch.bfloat16, "tokens")


def test_an_inference_call_between_the_passes_leaves_gradients_and_masks_alone():
    layer, g = _layer(96, 160, torch.bfloat16, 4, dropout=0.5)
    x, delta, dy, other = (torch.randn(n, 96, device="cuda", generator=g).bfloat16() for n in (48, 48, 48, 200))
    layer.forward(x, delta=delta)
    keep = rr.words(48, 96, layer.seed, 0, "cuda") >= 2 ** 31
    layer.forward(other, keep=False, delta=other)
    got = layer.backward(dy)
    p, want = _exact(layer, x, delta, keep)
    want.backward(dy.double())
    for k in got:
        _close(got[k], p[k].grad, torch.bfloat16, k)


def _eight(y):
    """Rows in 8 bits, as the values they stand for, in 64 bits."""
    scale = y.abs().amax(1, keepdim=True).clamp_min(rr.LEAST) / rr.TOP
    v = y / scale
    step = 2 * rr.half_step(v)
    return torch.round(v / step) * step * scale


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("tokens,model,hidden", SIZES)
def test_eight_bit_sublayer(tokens, model, hidden, add, dtype):
    layer, g = _layer(model, hidden, dtype, tokens)
    eight = layer.eight_bit()
    x, delta = (torch.randn(tokens, model, device="cuda", generator=g).to(dtype) for _ in range(2))
    y = eight.forward(x, delta=delta if add else None)
    assert dg.hgemm_last_device_status() == dg.DGEMM_OK
    s = x.double() + delta.double() if add else x.double()
    w = {}
    for k in ("wg", "wu", "wd"):
        w[k] = getattr(eight, k).double() * getattr(eight, "s" + k[1:]).double()[:, None]
        _close(w[k], _eight(getattr(layer, k).double()), dtype, k, 2.0 ** -8)     # ties alone may fall otherwise
    n = _eight(s * (s.square().mean(1, keepdim=True) + 1e-5).rsqrt() * layer.gamma.double())
    gate = n @ w["wg"].t()
    h = _eight((gate * torch.sigmoid(gate) * (n @ w["wu"].t())).to(dtype).double())
    part = h @ w["wd"].t()
    error = (y.double() - (s + part + layer.bd.double())).norm()
    assert float(error) <= 2.0 ** -5 * float(part.norm()) + 3 * U[dtype] * float(y.double().norm())
    # against the 16-bit sublayer: four roundings to e4m3 lie on a path (n, weights, h, weights), each below 2^-4 of its value
    full = layer.forward(x, keep=False, delta=delta if add else None)
    assert float((y.double() - full.double()).norm()) <= 4 * 2.0 ** -4 * float(part.norm()) + 9 * U[dtype] * float(full.double().norm())


def test_the_run_of_a_token_in_a_graph():
    """Norm to 8 bits, gated projections, rows to 8 bits, product: captured once and replayed on new tokens."""
    layer, g = _layer(512, 1024, torch.bfloat16, 3)
    eight = layer.eight_bit()
    xs = torch.randn(5, 512, device="cuda", generator=g).bfloat16()
    x = xs[:1].clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        want = [eight.forward(xs[i:i + 1]).clone() for i in range(5)]
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            y = eight.forward(x)
    for i in range(5):
        x.copy_(xs[i:i + 1])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want[i])


def test_refusals():
    for bad in (dict(norm="batch"), dict(dropout=1.0), dict(dropout=-0.1)):
        with pytest.raises(ValueError):
            FeedForward(64, 64, **bad)
    layer = FeedForward(64, 64)
    x = torch.zeros(2, 64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError):
        layer.forward(x, delta=x)
    with pytest.raises(ValueError):
        layer.eight_bit()
    with pytest.raises(RuntimeError):
        FeedForward(64, 64, norm="rms").backward(x)


def test_the_command_runs():
    import subprocess
    import sys
    run = subprocess.run([sys.executable, "-m", "paper_2003_00532_b200.feed_forward", "--model", "128", "--hidden", "256", "--tokens", "64", "--steps", "2",
                          "--norm", "rms", "--dropout", "0.1"], capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and "answering in 8 bits" in run.stdout, run.stdout + run.stderr
