"""Dropout behind the feed-forward sublayer with layer norm, both passes, against torch's differentiation in 64 bits. Needs a B200. Tolerance as in
test_gpu_feed_forward_rms: nine roundings to 16 bits on any path, relative in the 2-norm; and one more for the residual's gradient, which layer
norm's backward pass adds to a rounded value."""
import pytest
import torch

import hgemm_reference as ref
import rows_reference as rr
from paper_2003_00532_b200.feed_forward import FeedForward
from test_gpu_feed_forward import _exact

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("tokens,model,hidden", [(1, 64, 100), (37, 200, 333), (300, 520, 1000)])
def test_layer_norm_and_dropout(tokens, model, hidden, dtype):
    layer = FeedForward(model, hidden, dtype=dtype, seed=tokens, dropout=0.25)
    g = torch.Generator(device="cuda").manual_seed(5)
    layer.bd.add_(torch.randn(model, device="cuda", generator=g) * 0.2)
    x, dy = (torch.randn(tokens, model, device="cuda", generator=g).to(dtype) for _ in range(2))
    for use in range(2):
        y, got = layer.forward(x), layer.backward(dy)
        keep = rr.words(tokens, model, layer.seed, use, "cuda") >= 2 ** 30
        p, whole = _exact(layer, x)                   # x + f
        want = p["x"] + (whole - p["x"]) * keep / 0.75
        want.backward(dy.double())
        assert float((y.double() - want).detach().norm()) <= 9 * ref.U[dtype] * float(want.detach().norm())
        for k in got:
            rel = float((got[k].double() - p[k].grad).norm() / p[k].grad.norm())
            assert rel <= 10 * ref.U[dtype], f"{k}: {rel:.3g}"
