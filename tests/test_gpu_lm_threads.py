"""The 16-bit products and layer norm called from several host threads at once, each on a stream of its own. Needs a B200.
Integer data: every result is exact."""
import threading

import pytest
import torch

import paper_2003_00532_b200 as dg
from test_gpu_hgemm import _draw, _gen

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("threads", [2, 6])
def test_threads_on_their_own_streams(threads, dtype):
    g = _gen(threads)
    M, N, K = 20, 301, 4000       # cut tiles and rewritten operands
    A, B, C = _draw(g, M, K, dtype, 1.0, True, 3), _draw(g, N, K, dtype, 1.0, True, 1), _draw(g, N, K, dtype, 1.0, True, 1)
    dD, G, U = (_draw(g, M, N, dtype, 1.0, True, 1) for _ in range(3))
    X = _draw(g, 600, 1000, dtype, 1.0, True)
    mean, rstd = torch.zeros(600, device="cuda"), torch.ones(600, device="cuda")

    def outputs():
        e = lambda *s, t=dtype: torch.full(s, float("nan"), dtype=t, device="cuda")   # noqa: E731
        return {"D": e(M, N), "dA": e(M, K), "dB": e(N, K), "db": e(N, t=torch.float32), "dX": e(M, K), "dWg": e(N, K),
                "dx": e(600, 1000), "dga": e(1000, t=torch.float32), "dbe": e(1000, t=torch.float32)}

    def calls(o, stream):
        dg.hgemm_epilogue(A, B, o["D"], transb=True, stream=stream)
        dg.hgemm_epilogue_bwd(A, B, dD, act=dg.HGEMM_ACT_RELU, preact=G, dA=o["dA"], dB=o["dB"], dbias=o["db"], transb=True, stream=stream)
        dg.hgemm_gated_bwd(A, B, C, G, U, dD, act=dg.HGEMM_ACT_RELU, dX=o["dX"], dWg=o["dWg"], transw=True, stream=stream)
        dg.layernorm_bwd(X, None, mean, rstd, X, dX=o["dx"], dgamma=o["dga"], dbeta=o["dbe"], stream=stream)

    want = outputs()
    calls(want, torch.cuda.current_stream())
    assert torch.equal(want["D"], (A.double() @ B.double().t()).to(dtype))
    assert torch.equal(want["db"].double(), (dD.double() * (G.double() > 0)).sum(0))
    torch.cuda.synchronize()
    sets = [[outputs() for _ in range(6)] for _ in range(threads)]
    torch.cuda.synchronize()
    failed = []

    def work(mine):
        try:
            stream = torch.cuda.Stream()
            for _ in range(4):
                for o in mine:
                    calls(o, stream)
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
            for name in want:
                assert torch.equal(o[name], want[name]), name
