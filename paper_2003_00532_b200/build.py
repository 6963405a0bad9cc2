"""Builds ``libdgemm.so`` in-tree with nvcc for sm_100a (cross-compiles without a GPU)."""
from __future__ import annotations

import glob
import os
import shlex
import subprocess
import sys
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libdgemm.so")
EXT = os.path.join(HERE, "_marshal.so")  # compiled argument marshalling (csrc/binding_ext.cpp)
EXT_SOURCE = os.path.join(CSRC, "binding_ext.cpp")
SOURCES = [os.path.join(CSRC, name) for name in ("dgemm_api.cu", "sgemm_api.cu", "hgemm_api.cu", "hgemm_plain_f16.cu", "hgemm_plain_bf16.cu",
                                                "hgemm_gated_f16.cu", "hgemm_gated_bf16.cu", "hgemm_token.cu", "layernorm.cu")]
# every source, header and public header: an edit to any of them makes the built library stale
DEPS = sorted(glob.glob(os.path.join(CSRC, "*.cu")) + glob.glob(os.path.join(CSRC, "*.cuh")) +
              glob.glob(os.path.join(CSRC, "*.h")) + [EXT_SOURCE] + glob.glob(os.path.join(os.path.dirname(HERE), "include", "*.h")))

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-Xcompiler", "-fPIC", "-Xcompiler", "-fvisibility=hidden", "-cudart", "static",
]


def nvcc_path() -> str:
    cand = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "bin", "nvcc")
    return cand if os.path.exists(cand) else "nvcc"


def is_stale() -> bool:
    if not os.path.exists(LIB) or not os.path.exists(EXT):
        return True
    t = min(os.path.getmtime(LIB), os.path.getmtime(EXT))
    return any(os.path.getmtime(d) > t for d in DEPS)


# What ptxas must report for the kernels whose speed hangs on their register allocation: (substring
# of the mangled name, registers per thread at launch, most bytes of spill stores tolerated). The
# warp-specialised kernels redistribute a pool of threads x registers with setmaxnreg, so another
# launch count changes the consumers' budget; the 8192^3 figure was measured with exactly these.
PTXAS_EXPECT = [
    ("dgemm_dmma_ws_kernelILb1ELi128ELb0ELb0EE", 168, 128),
    ("dgemm_dmma_ws_kernelILb1ELi64ELb0ELb0EE", 128, 128),
    ("dgemm_dmma_kernelILb1ELi64ELi64ELi128ELi0ELb0ELb0EE", 255, 64),
    ("hgemm_tc_kernelI13__nv_bfloat16Li2ELi256ELi1ELb0ELi0EE", 168, 0),
    ("hgemm_tc_kernelI13__nv_bfloat16Li2ELi256ELi1ELb1ELi4EE", 164, 0),
]


def check_ptxas(log: str) -> None:
    """Raises if the `-Xptxas -v` output in `log` departs from PTXAS_EXPECT (a toolchain that allocates
    registers differently would silently change the measured speed)."""
    import re
    found = {}
    current = None
    spill = 0
    for line in log.splitlines():
        m = re.search(r"Compiling entry function '([^']+)'", line)
        if m:
            current, spill = m.group(1), 0
            continue
        m = re.search(r"(\d+) bytes spill stores", line)
        if m and current:
            spill = int(m.group(1))
        m = re.search(r"Used (\d+) registers", line)
        if m and current:
            found[current] = (int(m.group(1)), spill)
            current = None
    problems = []
    for key, regs, max_spill in PTXAS_EXPECT:
        hits = [(name, v) for name, v in found.items() if key in name]
        if not hits:
            problems.append(f"{key}: not found in the ptxas output")
        for name, (r, sp) in hits:
            if r != regs or sp > max_spill:
                problems.append(f"{name}: {r} registers, {sp} bytes of spill stores; expected {regs} and at most {max_spill}")
    if problems:
        raise RuntimeError("ptxas resource usage changed:\n  " + "\n  ".join(problems))


def ext_command(out: str) -> list:
    """The compiler command of the marshalling module (C++ only, against the installed torch)."""
    import sysconfig

    import torch
    from torch.utils.cpp_extension import include_paths
    torch_lib = os.path.join(os.path.dirname(torch.__file__), "lib")
    cuda = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "include")
    inc = [*include_paths(), sysconfig.get_paths()["include"], cuda]
    return ["g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-fvisibility=hidden", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
            *(f"-isystem{d}" for d in inc), EXT_SOURCE, "-o", out, f"-L{torch_lib}", f"-Wl,-rpath,{torch_lib}",
            "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda"]


def build(force: bool = False, verbose: bool = False, check: bool = False) -> str:
    """Compile the library if it is missing or older than its sources; returns its path. With `check`
    the compile reports resource usage and fails if the hot kernels' registers or spills changed."""
    if force or is_stale():
        tmp = LIB + ".tmp.%d" % os.getpid()
        extra = shlex.split(os.environ.get("DGEMM_NVCC_FLAGS", ""))  # e.g. -D switches for experiments
        flags = [*NVCC_FLAGS, *extra, *(["-Xptxas", "-v"] if (verbose or check) else [])]
        with tempfile.TemporaryDirectory() as objs:
            # one compiler process per source, side by side
            jobs = []
            for src in SOURCES:
                obj = os.path.join(objs, os.path.basename(src) + ".o")
                log = open(obj + ".log", "w+")
                jobs.append((obj, log, subprocess.Popen([nvcc_path(), *flags, "-c", "-o", obj, src], cwd=CSRC, stdout=log,
                                                        stderr=subprocess.STDOUT, text=True)))
            ext_tmp, ext_log = EXT + ".tmp.%d" % os.getpid(), open(os.path.join(objs, "ext.log"), "w+")
            jobs.append((None, ext_log, subprocess.Popen(ext_command(ext_tmp), cwd=CSRC, stdout=ext_log, stderr=subprocess.STDOUT, text=True)))
            failed, text = False, ""
            for obj, log, proc in jobs:
                failed = proc.wait() != 0 or failed
                log.seek(0)
                text += log.read()
                log.close()
            if not failed:
                res = subprocess.run([nvcc_path(), *flags, "-shared", "-o", tmp, *(j[0] for j in jobs if j[0])], cwd=CSRC,
                                     capture_output=True, text=True)
                failed = res.returncode != 0
                text += res.stdout + res.stderr
        if verbose or failed:
            sys.stderr.write(text)
        if failed:
            raise RuntimeError("nvcc failed building libdgemm.so")
        if check and not extra:
            check_ptxas(text)
        os.replace(tmp, LIB)
        os.replace(ext_tmp, EXT)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
