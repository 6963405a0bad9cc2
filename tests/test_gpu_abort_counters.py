"""A timed-out call leaves nothing behind for the calls beside it and after it: the counters that join the parts of cut tiles
return to zero by themselves, and reading the status touches no other call's. Needs a B200. Nothing faults, traps or waits
without a limit: the producers of the timed-out calls skip their copies, and their waits end after 3 ms. Integer data: exact."""
import pytest
import torch

import paper_2003_00532_b200 as dg
from test_gpu_hgemm import _draw, _gen

pytestmark = pytest.mark.gpu

BF = torch.bfloat16
CUT = [(8, 512, 4096), (300, 700, 6000), (130, 257, 9000)]


def _problem(M, N, K, gated, seed=1):
    g = _gen(seed)
    A, B, C = (_draw(g, r, K, BF, 1.0, True) for r in (M, N, N))
    want = A.double() @ B.double().t()
    if gated:
        want = want * (A.double() @ C.double().t())

    def call(D):
        if gated:
            return dg.hgemm_gated(A, B, C, D, act=dg.HGEMM_ACT_NONE, transw=True)
        return dg.hgemm_epilogue(A, B, D, transb=True)

    return call, want.to(BF)


def _timed_out(call, D):
    dg.hgemm_set_test_drop_loads(3000)
    try:
        assert call(D) == dg.DGEMM_OK
    finally:
        dg.hgemm_set_test_drop_loads(0)


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("shape", CUT)
def test_the_next_call_is_right_before_the_status_is_read(shape, gated):
    assert dg.hgemm_plan(*shape, gated=gated)["span"] > 0
    call, want = _problem(*shape, gated)
    assert dg.hgemm_last_device_status() == dg.DGEMM_OK
    outs = [torch.full_like(want, float("nan")) for _ in range(4)]
    _timed_out(call, outs[0])
    for D in outs[1:]:
        call(D)
    torch.cuda.synchronize()
    assert all(torch.equal(D, want) for D in outs[1:])
    assert dg.hgemm_last_device_status() == dg.binding.DGEMM_ERR_TIMEOUT
    assert dg.hgemm_last_device_status() == dg.DGEMM_OK


@pytest.mark.parametrize("gated", [False, True])
def test_reading_the_status_leaves_calls_on_another_stream_alone(gated):
    first, _ = _problem(*CUT[0], gated)
    call, want = _problem(*CUT[1], gated, seed=2)
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    D = torch.empty(CUT[0][0], CUT[0][1], dtype=BF, device="cuda")
    outs = [torch.full_like(want, float("nan")) for _ in range(120)]
    torch.cuda.synchronize()
    for s in (a, b):                      # (scratch of both streams)
        with torch.cuda.stream(s):
            first(D)
            call(outs[0])
            s.synchronize()
    for round_ in range(5):
        with torch.cuda.stream(a):
            _timed_out(first, D)
        with torch.cuda.stream(b):
            for o in outs:
                call(o)
        assert dg.hgemm_last_device_status(a) == dg.binding.DGEMM_ERR_TIMEOUT      # while b's calls are in flight
        b.synchronize()
        assert all(torch.equal(o, want) for o in outs)
        assert dg.hgemm_last_device_status(b) == dg.DGEMM_OK
    torch.cuda.synchronize()
