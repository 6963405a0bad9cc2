"""What the feed-forward sublayer keeps between its passes and what it hands out. Needs a B200. Tolerance as in
``test_gpu_feed_forward``: eight roundings to 16 bits on any path, relative in the 2-norm."""
import pytest
import torch

from paper_2003_00532_b200.feed_forward import FeedForward
from test_gpu_feed_forward import U, _exact

pytestmark = pytest.mark.gpu


def _inputs(layer, tokens, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return tuple(torch.randn(tokens, layer.model, device="cuda", generator=g).to(layer.dtype) for _ in range(2))


def _check_gradients(layer, x, dy, got):
    p, want = _exact(layer, x)
    want.backward(dy.double())
    for name in got:
        rel = float((got[name].double() - p[name].grad).norm() / p[name].grad.norm())
        assert rel <= 8 * U[layer.dtype], f"{name}: {rel:.3g}"


@pytest.mark.parametrize("tokens,between", [(48, 48), (48, 7), (48, 200), (1, 1)])
@pytest.mark.parametrize("dtype", list(U))
def test_an_inference_call_between_the_passes_leaves_the_gradients_alone(tokens, between, dtype):
    layer = FeedForward(96, 160, dtype=dtype, seed=4)
    (x, dy), (other, _) = _inputs(layer, tokens, 5), _inputs(layer, between, 6)
    layer.forward(x)
    layer.forward(other, keep=False)
    _check_gradients(layer, x, dy, layer.backward(dy))


def test_gradients_are_those_of_the_last_kept_pass():
    layer = FeedForward(96, 160, seed=4)
    for tokens, seed in ((40, 1), (40, 2), (9, 3), (300, 4), (40, 5)):
        x, dy = _inputs(layer, tokens, seed)
        layer.forward(x)
        _check_gradients(layer, x, dy, layer.backward(dy))


def test_results_stay_as_they_were_handed_out():
    layer = FeedForward(96, 160, seed=4)
    (x, dy), (x2, dy2) = _inputs(layer, 40, 1), _inputs(layer, 40, 2)
    held = []
    for a, b in ((x, dy), (x2, dy2)):
        y = layer.forward(a)
        grads = layer.backward(b)
        z = layer.forward(a, keep=False)
        held.append((y, y.clone(), z, z.clone(), grads, {k: v.clone() for k, v in grads.items()}))
    for y, y0, z, z0, grads, grads0 in held:
        assert torch.equal(y, y0) and torch.equal(z, z0) and torch.equal(y, z)
        assert all(torch.equal(grads[k], grads0[k]) for k in grads0)


def test_memory_does_not_grow_with_the_number_of_sizes_seen():
    layer = FeedForward(96, 160, seed=4)
    layer.backward(torch.zeros_like(layer.forward(_inputs(layer, 64, 0)[0])))
    layer.forward(_inputs(layer, 64, 0)[0], keep=False)
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    for tokens in range(1, 64):
        x, dy = _inputs(layer, tokens, tokens)
        layer.forward(x)
        layer.backward(dy)
        layer.forward(x, keep=False)
    del x, dy
    torch.cuda.synchronize()
    # at most the last input, kept for a further backward pass
    assert torch.cuda.memory_allocated() - before <= 64 * layer.model * 2


def test_backward_needs_a_kept_pass():
    layer = FeedForward(96, 160, seed=4)
    x, dy = _inputs(layer, 4, 1)
    layer.forward(x, keep=False)
    with pytest.raises(RuntimeError):
        layer.backward(dy)


def test_a_failed_pass_is_not_kept():
    layer = FeedForward(96, 160, seed=4)
    x, dy = _inputs(layer, 4, 1)
    layer.forward(x)
    with pytest.raises(TypeError):
        layer.forward(x.float())
    with pytest.raises(RuntimeError):
        layer.backward(dy)
