"""Passes of the feed-forward sublayer that are captured into CUDA graphs, with larger passes between capture and replay. Needs a B200. Every
comparison is between equal bits, but for the sums in ``test_every_replay_drops_others``: 60 binary32 additions of exact values, each off by
2^-24 of a partial sum."""
import pytest
import torch

import rows_reference as rr
from paper_2003_00532_b200.feed_forward import FeedForward

pytestmark = pytest.mark.gpu

MODEL, HIDDEN = 256, 640


def _capture(call):
    """(graph, result) of `call`, captured on a stream of its own."""
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream), torch.cuda.graph(graph, stream=stream):
        result = call()
    torch.cuda.synchronize()
    return graph, result


def _others():
    """Tensors of one value in every size that a freed buffer could be given to next."""
    return [torch.full((n,), 7.0, device="cuda") for n in [128] * 64 + [256] * 64 + [1024] * 64 + [64 * 1024] * 16 + [1 << 19] * 8]


def _intact(others):
    return all(bool((t == 7.0).all()) for t in others)


@pytest.mark.parametrize("kind", ["16 bits", "8 bits", "layer norm"])
@pytest.mark.parametrize("warm", [True, False])
def test_a_token_is_replayed_after_larger_prompts(kind, warm):
    def pass_of(layer):
        return layer.eight_bit().forward if kind == "8 bits" else lambda x: layer.forward(x, keep=False)

    run, warmed = (pass_of(FeedForward(MODEL, HIDDEN, seed=1, norm="layer" if kind == "layer norm" else "rms")) for _ in range(2))
    xs = torch.randn(300, MODEL, device="cuda", generator=torch.Generator(device="cuda").manual_seed(2)).bfloat16()
    x, want = xs[:1].clone(), None
    warmed(x)   # (kernels are loaded; another object's buffers)
    if warm:
        want = [run(xs[i:i + 1]) for i in range(4)]
    graph, y = _capture(lambda: run(x))
    prompts = [run(xs[:n]) for n in (8, 300)]
    others = _others()
    if not warm:
        want = [run(xs[i:i + 1]) for i in range(4)]
    for i in range(4):
        x.copy_(xs[i:i + 1])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want[i])
        assert torch.equal(run(xs[:8]), prompts[0]) and torch.equal(run(xs), prompts[1])   # prompts and tokens in turn
    assert _intact(others)


@pytest.mark.parametrize("norm", ["layer", "rms"])
def test_a_training_pass_is_replayed_after_a_larger_one(norm):
    layer = FeedForward(MODEL, HIDDEN, seed=1, norm=norm)
    g = torch.Generator(device="cuda").manual_seed(3)
    xs, dys = (torch.randn(3, 40, MODEL, device="cuda", generator=g).bfloat16() for _ in range(2))
    big, dbig = (torch.randn(500, MODEL, device="cuda", generator=g).bfloat16() for _ in range(2))
    x, dy = xs[0].clone(), dys[0].clone()

    def both(a, b):
        y = layer.forward(a)
        return dict(layer.backward(b), y=y)

    want = [both(a, b) for a, b in zip(xs, dys)]
    graph, got = _capture(lambda: both(x, dy))
    large = both(big, dbig)
    others = _others()
    for a, b, w in zip(xs, dys, want):
        x.copy_(a)
        dy.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        for k in w:
            assert torch.equal(got[k], w[k]), k
        again = both(big, dbig)
        for k in again:
            assert torch.equal(again[k], large[k]), k
    assert _intact(others)


def test_a_forward_pass_and_its_gradients_in_two_graphs():
    """The gradients' graph reads what the forward pass's graph has kept, with other passes captured and run between them."""
    layer = FeedForward(MODEL, HIDDEN, seed=1, norm="rms")
    g = torch.Generator(device="cuda").manual_seed(4)
    x, dy, delta = (torch.randn(24, MODEL, device="cuda", generator=g).bfloat16() for _ in range(3))
    other = torch.randn(333, MODEL, device="cuda", generator=g).bfloat16()
    y = layer.forward(x, delta=delta)
    want = dict(layer.backward(dy), y=y)
    first, y = _capture(lambda: layer.forward(x, delta=delta))
    second, got = _capture(lambda: layer.backward(dy))
    layer.forward(other)
    layer.backward(other)
    others = _others()
    for t in [y, *got.values()]:
        t.zero_()
    first.replay()
    layer.forward(other, keep=False)
    second.replay()
    torch.cuda.synchronize()
    got["y"] = y
    for k in want:
        assert torch.equal(got[k], want[k]), k
    assert _intact(others)


@pytest.mark.parametrize("norm", ["layer", "rms"])
def test_every_replay_drops_others(norm):
    """Two captured training passes with dropout, and others between their replays: a mask of its own each time, the same in its gradients."""
    layer = FeedForward(MODEL, HIDDEN, seed=1, norm=norm, dropout=0.5)
    g = torch.Generator(device="cuda").manual_seed(5)
    x, dy = (torch.randn(60, MODEL, device="cuda", generator=g).bfloat16() for _ in range(2))

    def both():
        y = layer.forward(x)
        return y, layer.backward(dy)["bd"]

    seen = []

    def check(y, bd):
        torch.cuda.synchronize()
        dropped = y == x     # (what is kept is nowhere so small that it is lost in the addition, or few times)
        for mask in seen:
            assert 0.4 < float((dropped == mask).float().mean()) < 0.6
        seen.append(dropped)
        assert 0.45 < float(dropped.float().mean()) < 0.55
        return dropped

    def exactly(y, bd, use):
        keep = rr.words(60, MODEL, layer.seed, use, "cuda") >= 2 ** 31
        dropped = check(y, bd)
        assert bool(dropped[~keep].all()) and float(dropped[keep].float().mean()) < 0.05
        parts = dy.double() * 2 * keep
        assert bool(((bd.double() - parts.sum(0)).abs() <= 60 * 2.0 ** -24 * parts.abs().sum(0)).all())

    exactly(*both(), 0)
    graphs = [_capture(both) for _ in range(2)]
    for k, which in enumerate((0, 1, 1, 0)):
        graph, result = graphs[which]
        graph.replay()
        exactly(*result, (1 << 62) + k + 1)
        exactly(*both(), k + 1)
