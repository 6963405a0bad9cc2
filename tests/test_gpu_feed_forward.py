"""The feed-forward sublayer that runs layer norm, the gated projections and the product with bias and residual
together, against the same sublayer in 64 bits with torch's own differentiation. Needs a B200.

Tolerance: every intermediate (n, gate, up, h, dh, dn and the outputs) is rounded once to 16 bits, an error of u times
its size with independent signs; at most eight such roundings lie on any path from an input to a gradient, so the
relative error of a whole matrix (2-norm) stays below 8 u (u = 2^-8 bfloat16, 2^-11 binary16)."""
import pytest
import torch

import paper_2003_00532_b200 as dg
from paper_2003_00532_b200.feed_forward import FeedForward

pytestmark = pytest.mark.gpu

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def _exact(layer, x):
    p = {k: getattr(layer, k).double().requires_grad_() for k in ("gamma", "beta", "wg", "wu", "wd", "bd")}
    p["x"] = x.double().requires_grad_()
    d = p["x"] - p["x"].mean(1, keepdim=True)
    n = d / (d.square().mean(1, keepdim=True) + 1e-5).sqrt() * p["gamma"] + p["beta"]
    g = n @ p["wg"].t()
    y = p["x"] + (g * torch.sigmoid(g) * (n @ p["wu"].t())) @ p["wd"].t() + p["bd"]
    return p, y


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("tokens,model,hidden", [(1, 64, 100), (2, 256, 512), (37, 200, 333), (300, 520, 1000), (1024, 1024, 2048)])
def test_sublayer_and_gradients(tokens, model, hidden, dtype):
    layer = FeedForward(model, hidden, dtype=dtype, seed=tokens)
    g = torch.Generator(device="cuda").manual_seed(5)
    layer.gamma.add_(torch.randn(model, device="cuda", generator=g) * 0.2)
    layer.bd.add_(torch.randn(model, device="cuda", generator=g) * 0.2)
    x = torch.randn(tokens, model, device="cuda", generator=g).to(dtype)
    dy = torch.randn(tokens, model, device="cuda", generator=g).to(dtype)
    y = layer.forward(x)
    got = {k: v.clone() for k, v in layer.backward(dy).items()}
    assert dg.hgemm_last_device_status() == dg.DGEMM_OK
    p, want = _exact(layer, x)
    want.backward(dy.double())
    pairs = {"y": (y, want.detach())}
    pairs.update({k: (got[k], p[k].grad) for k in got})
    for name, (a, b) in pairs.items():
        rel = float((a.double() - b).norm() / b.norm())
        assert rel <= 8 * U[dtype], f"{name}: {rel:.3g}"


def test_training_lowers_the_loss_and_tokens_agree_with_the_batch():
    layer, teacher = FeedForward(256, 512, seed=1), FeedForward(256, 512, seed=2)
    x = torch.randn(512, 256, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3)).to(layer.dtype)
    target = teacher.forward(x, keep=False).clone()
    losses = [layer.step(x, target, 0.05) for _ in range(15)]
    assert losses[-1] < 0.9 * losses[0]
    batch = layer.forward(x[:6], keep=False).clone()
    rows = torch.cat([layer.forward(x[i:i + 1], keep=False).clone() for i in range(6)])
    assert float((rows.double() - batch.double()).norm() / batch.double().norm()) <= 8 * U[layer.dtype]
