"""Products of one and two rows around the lengths where the tokens reach 48 KB of shared memory, the most that a kernel
may ask for without raising its limit, and where they no longer fit at all. Needs a B200.

The limit belongs to the kernel and stays raised, so the lengths run in ascending order in a process of their own: no
longer sum has come before."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

HERE = os.path.dirname(os.path.abspath(__file__))
PROGRAM = """
import sys
sys.path[:0] = {paths!r}
import hgemm_reference as ref
import test_gpu_hgemm as t
for M, lengths in ((1, (24536, 24544, 24552, 24573, 24576, 24577, 30000, 81920, 81928)),
                   (2, (12248, 12256, 12264, 12285, 12288, 12289, 20000, 40960, 40968))):
    for K in lengths:
        for dtype in t.TYPES:
            t._linear_case(M, 70, K, dtype, False, True, ref.NONE, True, True, True, seed=K, integer=True, pad=-K % 8)
            t._gated_case(M, 70, K, dtype, True, ref.SILU, True, seed=K, pad=-K % 8)
print("all lengths done")
"""


def test_lengths_where_shared_memory_needs_a_raised_limit():
    run = subprocess.run([sys.executable, "-c", PROGRAM.format(paths=[HERE, os.path.dirname(HERE)])], capture_output=True, text=True, timeout=600)
    assert run.returncode == 0 and "all lengths done" in run.stdout, run.stdout + run.stderr
