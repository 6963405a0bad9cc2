"""Graphs replayed after later calls that need more scratch memory than there was at capture. Needs a B200. Integer data:
results are exact, so every replay has to give the same bits."""
import pytest
import torch

import paper_2003_00532_b200 as dg

pytestmark = pytest.mark.gpu

BF = torch.bfloat16


def _ints(g, rows, cols, dtype=BF, pad=0):
    x = torch.empty(rows, cols + pad, dtype=dtype, device="cuda")[:, :cols]
    x.copy_(torch.randint(-3, 4, (rows, cols), device="cuda", generator=g))
    return x


def _decode_step(g):
    """Cut tiles (workspace, counters), rewritten operands, dG and dU in scratch, block sums: (call, outputs)."""
    A, B, D = _ints(g, 8, 4096), _ints(g, 512, 4096), torch.zeros(8, 512, dtype=BF, device="cuda")
    A1, B1, D1 = _ints(g, 9, 700, pad=1), _ints(g, 133, 700, pad=3), torch.zeros(9, 133, dtype=BF, device="cuda")
    G, U, dH, W = _ints(g, 40, 200), _ints(g, 40, 200), _ints(g, 40, 200), _ints(g, 200, 96)
    X, dX, dW = _ints(g, 40, 96), torch.zeros(40, 96, dtype=BF, device="cuda"), torch.zeros(200, 96, dtype=BF, device="cuda")
    mean, rstd, dga = torch.zeros(40, device="cuda"), torch.ones(40, device="cuda"), torch.zeros(96, device="cuda")
    Da, Db, Dc = (_ints(g, *s, dtype=torch.float64, pad=1) for s in ((300, 500), (500, 201), (300, 201)))

    def call():
        dg.hgemm_epilogue(A, B, D, transb=True)
        dg.hgemm_epilogue(A1, B1, D1, transb=True)
        dg.hgemm_gated_bwd(X, W, W, G, U, dH, act=dg.HGEMM_ACT_RELU, dX=dX, dWg=dW, transw=True)
        dg.layernorm_bwd(X, None, mean, rstd, X, dgamma=dga)
        Dc.zero_()
        dg.dgemm_f64(Da, Db, Dc)

    return call, (D, D1, dX, dW, dga, Dc)


def _larger(g):
    A, B, D = _ints(g, 700, 6000, pad=1), _ints(g, 3001, 6000, pad=1), torch.empty(700, 3001, dtype=BF, device="cuda")
    dg.hgemm_epilogue(A, B, D, transb=True)
    X, mean, rstd, dga = _ints(g, 3000, 12000), torch.zeros(3000, device="cuda"), torch.ones(3000, device="cuda"), torch.zeros(12000, device="cuda")
    dg.layernorm_bwd(X, None, mean, rstd, X, dgamma=dga)
    A, B, D = _ints(g, 16, 8192), _ints(g, 2048, 8192), torch.empty(16, 2048, dtype=BF, device="cuda")
    dg.hgemm_epilogue(A, B, D, transb=True)
    G, W, X = _ints(g, 2000, 1000), _ints(g, 1000, 500, pad=3), _ints(g, 2000, 500, pad=3)
    dg.hgemm_gated_bwd(X, W, W, G, G, G, act=dg.HGEMM_ACT_RELU, dX=torch.empty_like(X), dWg=torch.empty(1000, 500, dtype=BF, device="cuda"), transw=True)
    A, B = _ints(g, 1500, 1501, torch.float64, pad=2), _ints(g, 1501, 1503, torch.float64)
    dg.dgemm_f64(A, B, torch.zeros(1500, 1503, dtype=torch.float64, device="cuda"))


@pytest.mark.parametrize("streams", [1, 3])
def test_replay_after_larger_calls(streams):
    assert dg.dgemm_release_scratch() == dg.DGEMM_OK     # the pools start over, with no stream seen
    g = torch.Generator(device="cuda").manual_seed(streams)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        call, outs = _decode_step(g)
        others = [torch.cuda.Stream() for _ in range(streams - 1)]
        s.synchronize()
        for o in others:
            with torch.cuda.stream(o):
                call()
            o.synchronize()
        call()
        s.synchronize()
        want = [o.clone() for o in outs]
        assert torch.equal(want[0], want[0].round()) and float(want[0].float().abs().max()) > 0
        s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        call()
    for i in range(3):
        with torch.cuda.stream(s):
            _larger(g)
            s.synchronize()
            # memory that the device has free now, in the caller's hands
            held = [torch.full((n,), 7, dtype=torch.int32, device="cuda") for n in (1 << 16, 1 << 19, 1 << 22, 1 << 24)]
            for o in outs:
                o.zero_()
            s.synchronize()
            graph.replay()
            s.synchronize()
            for o, w in zip(outs, want):
                assert torch.equal(o, w)
            assert all(bool((h == 7).all()) for h in held)
            call()
            s.synchronize()
            for o, w in zip(outs, want):
                assert torch.equal(o, w)
    assert dg.hgemm_last_device_status(s) == dg.DGEMM_OK
    del graph
    torch.cuda.synchronize()
    assert dg.dgemm_release_scratch() == dg.DGEMM_OK
