"""Forward layer norm around the row lengths where a block's shared memory reaches 48 KB, the most that a kernel may ask
for without raising its limit. Needs a B200.

The limit belongs to the kernel and stays raised, so the lengths run in ascending order in a process of their own: no
longer row has come before."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

HERE = os.path.dirname(os.path.abspath(__file__))
PROGRAM = """
import sys
sys.path[:0] = {paths!r}
import torch
import test_gpu_layernorm as t
for cols in (5632, 5633, 5888, 5889, 6143, 6144, 6145, 6200):
    for dtype in t.TYPES:
        for rows in (3, 700):                    # rows spread over as many threads as possible, and 16 values per thread
            for odd in (False, True):            # rows of 16-byte vectors, and of single values
                pad = -cols % 8 + (3 if odd else 0)
                t._forward(rows, cols, dtype, seed=cols, pad=pad)
                t._backward(rows, cols, dtype, seed=cols, pad=pad)
print("all lengths done")
"""


def test_lengths_where_shared_memory_needs_a_raised_limit():
    run = subprocess.run([sys.executable, "-c", PROGRAM.format(paths=[HERE, os.path.dirname(HERE)])], capture_output=True, text=True, timeout=600)
    assert run.returncode == 0 and "all lengths done" in run.stdout, run.stdout + run.stderr
