"""A call that the CUDA runtime refuses leaves nothing behind for the next one. Needs a B200. In a process of its own: a stream
capture is spoilt by waiting for its stream, so that every launch into it is refused on the host; nothing reaches the GPU."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

PROGRAM = """
import sys
sys.path[:0] = [{root!r}]
import torch
import paper_2003_00532_b200 as dg
bf = torch.bfloat16
X, Y, W, D = (torch.ones(*s, dtype=bf, device="cuda") for s in ((64, 64), (64, 64), (64, 64), (64, 64)))
stats = torch.ones(64, device="cuda")
none, sums = torch.zeros(0, 64, dtype=bf, device="cuda"), torch.empty(64, device="cuda")
A, B, C = (torch.ones(70, 70, dtype=torch.float64, device="cuda") for _ in range(3))
A32, B32, C32 = (torch.ones(70, 70, device="cuda") for _ in range(3))
s = torch.cuda.Stream()
calls = {{
    "layernorm_fwd": lambda: dg.layernorm_fwd(X, None, None, Y, stream=s, check=False),
    "layernorm_bwd": lambda: dg.layernorm_bwd(X, None, stats, stats, X, dX=Y, stream=s, check=False),
    "layernorm_bwd, no rows": lambda: dg.layernorm_bwd(none, None, none[:, 0].float(), none[:, 0].float(), none, dgamma=sums, stream=s, check=False),
    "hgemm_epilogue": lambda: dg.hgemm_epilogue(X, W, D, stream=s, check=False),
    "hgemm_epilogue, one row": lambda: dg.hgemm_epilogue(X[:1], W, D[:1], transb=True, stream=s, check=False),
    "hgemm_epilogue, no terms": lambda: dg.hgemm_epilogue(X[:, :0], W[:0], D, stream=s, check=False),
    "hgemm_gated": lambda: dg.hgemm_gated(X, W, W, D, stream=s, check=False),
    "hgemm_epilogue_bwd": lambda: dg.hgemm_epilogue_bwd(X, W, D, dA=Y, stream=s, check=False),
    "hgemm_epilogue_bwd, no rows": lambda: dg.hgemm_epilogue_bwd(none, W, none, dbias=sums, stream=s, check=False),
}}
for call in calls.values():
    assert call() == dg.DGEMM_OK
torch.cuda.synchronize()
dg.dgemm_f64(A, B, C)
dg.sgemm_f32(A32, B32, C32)
for name, call in calls.items():
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        graph.capture_begin(capture_error_mode="relaxed")
        try:
            s.synchronize()
        except RuntimeError:
            pass
        rc = call()
        try:
            graph.capture_end()
        except RuntimeError:
            pass
    assert rc == dg.binding.DGEMM_ERR_CUDA, (name, rc)
    assert dg.dgemm_f64(A, B, C, check=False) == dg.DGEMM_OK, name + ": dgemm_f64 after it"
    assert dg.sgemm_f32(A32, B32, C32, check=False) == dg.DGEMM_OK, name + ": sgemm_f32 after it"
    assert call() == dg.DGEMM_OK, name
torch.cuda.synchronize()
print("all calls done")
"""


def test_the_next_call_does_not_report_an_earlier_error():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    run = subprocess.run([sys.executable, "-c", PROGRAM.format(root=root)], capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and "all calls done" in run.stdout, run.stdout + run.stderr
