"""The scratch pool's host logic against a fake CUDA runtime (tests/fake_cuda): what a captured graph refers to stays
allocated. No GPU."""
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2003_00532_b200", "csrc")


@pytest.mark.parametrize("program", ["scratch_pool_captured"])
def test_pool(program, tmp_path):
    out = str(tmp_path / program)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-pthread", "-I", os.path.join(HERE, "fake_cuda"), "-I", CSRC,
                    os.path.join(HERE, program + ".cpp"), "-o", out], check=True)
    run = subprocess.run([out], capture_output=True, text=True, timeout=60)
    assert run.returncode == 0 and run.stdout == "ok\n", run.stdout + run.stderr
