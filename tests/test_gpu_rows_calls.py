"""RMS norm, rows in 8 bits, dropout and the products of 8-bit operands as programs call them: from several threads at once, captured beside
larger calls and replayed, in matrices of more than 2^31 values. Needs a B200. Every comparison is between equal bits, or with the bounds
of ``rows_reference``."""
import threading

import pytest
import torch

import hgemm_reference as ref
import paper_2003_00532_b200 as dg
import rows_reference as rr
from test_gpu_hgemm import _gen

pytestmark = pytest.mark.gpu

BF = torch.bfloat16


def _inputs(rows, model, hidden, seed):
    """A sublayer's worth of calls; odd widths, so that operands are rewritten into scratch memory and products cut into parts."""
    g = _gen(seed)
    n = lambda *s, t=BF: torch.randn(*s, device="cuda", generator=g).to(t)   # noqa: E731
    q = lambda *s: (torch.randn(*s, device="cuda", generator=g) * 0.5).to(rr.E4M3)   # noqa: E731
    return {"x": n(rows, model), "r": n(rows, model), "gamma": n(model), "wg": q(hidden, model), "wu": q(hidden, model), "wd": q(model, hidden),
            "dy": n(rows, model), "ds": n(rows, model)}


def _outputs(i):
    rows, model = i["x"].shape
    hidden = i["wg"].shape[0]
    e = lambda *s, t=BF: torch.empty(*s, dtype=t, device="cuda")   # noqa: E731
    f = torch.float32
    return {"s": e(rows, model), "n": e(rows, model, t=rr.E4M3), "sn": e(rows, t=f), "rstd": e(rows, t=f), "h": e(rows, hidden),
            "q": e(rows, hidden, t=rr.E4M3), "sq": e(rows, t=f), "y": e(rows, model), "d": e(rows, model), "dx": e(rows, model), "dg": e(model, t=f),
            "dd": e(rows, model)}


def _run(i, o, **on):
    dg.rmsnorm_fwd_e4m3(i["x"], i["gamma"], o["n"], o["sn"], residual=i["r"], sum=o["s"], rstd=o["rstd"], **on)
    dg.qgemm_gated(o["n"], i["wg"], i["wu"], o["h"], x_scale=o["sn"], act=dg.HGEMM_ACT_SILU, **on)
    dg.quantize_rows_e4m3(o["h"], o["q"], o["sq"], **on)
    dg.qgemm_epilogue(o["q"], i["wd"], o["y"], a_scale=o["sq"], residual=o["s"], **on)
    dg.dropout_fwd(o["y"], o["d"], 0.3, 5, 6, residual=o["s"], **on)
    dg.rmsnorm_bwd(o["s"], i["gamma"], o["rstd"], i["dy"], dsum=i["ds"], dX=o["dx"], dgamma=o["dg"], **on)
    dg.dropout_bwd(o["dx"], o["dd"], 0.3, 5, 6, **on)


def _same(o, want):
    for k in want:
        a, b = (t.view(torch.uint8) for t in (o[k].contiguous(), want[k].contiguous()))
        assert torch.equal(a, b), k


@pytest.mark.parametrize("rows,model,hidden", [(1, 515, 1001), (40, 1001, 4003), (700, 515, 1001)])
def test_threads_on_their_own_streams(rows, model, hidden):
    i = _inputs(rows, model, hidden, rows)
    want = _outputs(i)
    _run(i, want)
    sets = [[_outputs(i) for _ in range(3)] for _ in range(4)]
    torch.cuda.synchronize()
    failed = []

    def work(mine):
        try:
            stream = torch.cuda.Stream()
            for _ in range(4):
                for o in mine:
                    _run(i, o, stream=stream)
            stream.synchronize()
            if dg.hgemm_last_device_status(stream) != dg.DGEMM_OK:
                failed.append("status")
        except Exception as e:   # noqa: BLE001  (reported by the main thread)
            failed.append(repr(e))

    pool = [threading.Thread(target=work, args=(s,)) for s in sets]
    for t in pool:
        t.start()
    for t in pool:
        t.join()
    torch.cuda.synchronize()
    assert not failed
    for mine in sets:
        for o in mine:
            _same(o, want)


def test_two_graphs_and_a_larger_call_between():
    """Two captured runs share the library's scratch memory; a larger eager call makes it grow before they are replayed, in either order and
    on two streams one after the other."""
    small, other, large = _inputs(40, 1001, 4003, 1), _inputs(33, 515, 1001, 2), _inputs(900, 1001, 4003, 3)
    want = [_outputs(small), _outputs(other)]
    _run(small, want[0])
    _run(other, want[1])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = [_outputs(small), _outputs(other)]
    graphs = []
    with torch.cuda.stream(s):
        for i, o in zip((small, other), got):
            _run(i, o)
            s.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=s):
                _run(i, o)
            graphs.append(graph)
    torch.cuda.synchronize()
    big = _outputs(large)
    _run(large, big)
    torch.cuda.synchronize()
    for order in ((0, 1), (1, 0), (0, 0, 1, 1)):
        for o in got:
            for t in o.values():
                t.view(torch.uint8).fill_(0x55)
        for k in order:
            graphs[k].replay()
        torch.cuda.synchronize()
        _same(got[0], want[0])
        _same(got[1], want[1])
    assert dg.hgemm_last_device_status() == dg.DGEMM_OK
    again = _outputs(large)
    _run(large, again)
    _same(again, big)


@pytest.mark.parametrize("cols", [4096, 4099, 9001])
def test_norms_of_more_than_2_to_the_31_values(cols):
    """The last rows of matrices whose offsets pass 32 bits, and a sum over all of them."""
    rows = 2 ** 31 // cols + 300
    X = torch.empty(rows, cols, dtype=BF, device="cuda")
    X.copy_(torch.randn(1, cols, device="cuda", generator=_gen(1)).to(BF).expand(rows, cols))
    X[-7:] = torch.randn(7, cols, device="cuda", generator=_gen(2)).to(BF)
    Y, r = torch.empty_like(X), torch.empty(rows, device="cuda")
    dg.rmsnorm_fwd(X, None, Y, residual=X, sum=None, rstd=r)
    part = slice(rows - 300, rows)
    _, y, rstd = rr.rms(X[part], X[part], None, 1e-5)
    ref.assert_within(Y[part], y, rr.value_bound(y, BF), "Y")
    ref.assert_within(r[part], rstd, rr.VALUE * rstd, "rstd")
    Q, scale = torch.empty(rows, cols, dtype=rr.E4M3, device="cuda"), torch.empty(rows, device="cuda")
    dg.rmsnorm_fwd_e4m3(X, None, Q, scale)
    _, y, _ = rr.rms(X[part], None, None, 1e-5)
    rr.assert_eight(Q[part], scale[part], y)
    dg.quantize_rows_e4m3(X, Q, scale)
    rr.assert_eight(Q[part], scale[part], X[part].double(), value=0.0)
    del Q
    dga = torch.empty(cols, device="cuda")
    dY = torch.zeros_like(X)
    dY[-300:] = torch.randn(300, cols, device="cuda", generator=_gen(3)).to(BF)
    dg.rmsnorm_bwd(X, None, r, dY, dX=Y, dgamma=dga)
    want = rr.rms_grad(X[part], None, r[part], dY[part], None)
    ref.assert_within(Y[part], *want["dX"], "dX")
    ref.assert_within(dga, *want["dgamma"], "dgamma")
    assert bool((Y[:-300] == 0).all())


def test_products_of_more_than_2_to_the_31_bytes():
    M, N, K = 70001, 8, 32768
    A = torch.zeros(M, K, dtype=torch.uint8, device="cuda").view(rr.E4M3)
    A[-5:] = (torch.randn(5, K, device="cuda", generator=_gen(1)) * 0.5).to(rr.E4M3)
    B = (torch.randn(N, K, device="cuda", generator=_gen(2)) * 0.5).to(rr.E4M3)
    D = torch.empty(M, N, dtype=BF, device="cuda")
    dg.qgemm_epilogue(A, B, D)
    assert dg.hgemm_last_device_status() == dg.DGEMM_OK
    d, bound, _, _ = rr.linear8(A[-5:], B, None, None, None, ref.NONE, None, BF)
    ref.assert_within(D[-5:], d, bound, "D")
    assert bool((D[:-5] == 0).all())
    # the long matrix as weights of one token and of three
    for rows in (1, 3):
        D = torch.empty(rows, M, dtype=BF, device="cuda")
        dg.qgemm_epilogue(B[:rows], A, D)
        d, bound, _, _ = rr.linear8(B[:rows], A[-5:], None, None, None, ref.NONE, None, BF)
        ref.assert_within(D[:, -5:], d, bound, "D")
        assert bool((D[:, :-5] == 0).all())


def test_another_stream_without_a_wait():
    """All calls run on the stream that they are given, none on the current one."""
    i = _inputs(40, 1001, 4003, 5)
    want, got = _outputs(i), _outputs(i)
    _run(i, want)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        _run(i, got)
    s.synchronize()
    _same(got, want)
