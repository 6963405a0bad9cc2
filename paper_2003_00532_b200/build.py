"""Builds ``libdgemm.so`` in-tree with nvcc for sm_100a (cross-compiles without a GPU), and ``_marshal.so``, the compiled
argument marshalling of some Python entry points, with g++ against the installed torch. Nothing in the library uses torch:
without torch it is built alone, and those entry points say what is missing when they are first used."""
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
EXT_STAMP = EXT + ".torch"  # the torch and the Python that it was built against
SOURCES = [os.path.join(CSRC, name) for name in ("dgemm_api.cu", "sgemm_api.cu", "hgemm_api.cu", "hgemm_plain_f16.cu", "hgemm_plain_bf16.cu",
                                                "hgemm_gated_f16.cu", "hgemm_gated_bf16.cu", "hgemm_token.cu", "qgemm_token.cu", "qgemm_plain_f16.cu", "qgemm_plain_bf16.cu",
                                                "qgemm_gated_f16.cu", "qgemm_gated_bf16.cu", "layernorm.cu", "rmsnorm.cu", "dropout.cu")]
HEADERS = sorted(glob.glob(os.path.join(CSRC, "*.cuh")) + glob.glob(os.path.join(CSRC, "*.h")) +
                 glob.glob(os.path.join(os.path.dirname(HERE), "include", "*.h")))
# every source, header and public header: an edit to any of them makes what is built from them stale
LIB_DEPS = sorted(glob.glob(os.path.join(CSRC, "*.cu"))) + HEADERS
EXT_DEPS = [EXT_SOURCE] + HEADERS
DEPS = LIB_DEPS + [EXT_SOURCE]

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-Xcompiler", "-fPIC", "-Xcompiler", "-fvisibility=hidden", "-cudart", "static",
]


def nvcc_path() -> str:
    cand = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "bin", "nvcc")
    return cand if os.path.exists(cand) else "nvcc"


def _older(built: str, deps: list) -> bool:
    return not os.path.exists(built) or any(os.path.getmtime(d) > os.path.getmtime(built) for d in deps)


def torch_version() -> str | None:
    """The installed torch's version and this Python's, or None without torch."""
    import importlib.metadata
    import importlib.util
    if "torch" in sys.modules and sys.modules["torch"] is None or importlib.util.find_spec("torch") is None:
        return None
    return "torch %s, %s" % (importlib.metadata.version("torch"), sys.version.split()[0])


def lib_is_stale() -> bool:
    return _older(LIB, LIB_DEPS)


def ext_is_stale() -> bool:
    """Missing, older than its sources, or built against another torch or Python than the installed ones."""
    if _older(EXT, EXT_DEPS) or not os.path.exists(EXT_STAMP):
        return True
    with open(EXT_STAMP) as f:
        return f.read() != torch_version()


def is_stale() -> bool:
    return lib_is_stale() or (torch_version() is not None and ext_is_stale())


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


def _compile_all(commands: list) -> tuple:
    """Runs the commands side by side; (whether all succeeded, their output)."""
    jobs = []
    for cmd in commands:
        log = tempfile.TemporaryFile("w+")
        jobs.append((log, subprocess.Popen(cmd, cwd=CSRC, stdout=log, stderr=subprocess.STDOUT, text=True)))
    ok, text = True, ""
    for log, proc in jobs:
        ok = proc.wait() == 0 and ok
        log.seek(0)
        text += log.read()
        log.close()
    return ok, text


def build(force: bool = False, verbose: bool = False, check: bool = False) -> str:
    """Compile what is missing or older than its sources; returns the library's path. With `check`
    the compile reports resource usage and fails if the hot kernels' registers or spills changed."""
    do_lib = force or lib_is_stale()
    version = torch_version()
    do_ext = version is not None and (force or ext_is_stale())
    extra = shlex.split(os.environ.get("DGEMM_NVCC_FLAGS", ""))  # e.g. -D switches for experiments
    flags = [*NVCC_FLAGS, *extra, *(["-Xptxas", "-v"] if (verbose or check) else [])]
    lib_tmp, ext_tmp = LIB + ".tmp.%d" % os.getpid(), EXT + ".tmp.%d" % os.getpid()
    with tempfile.TemporaryDirectory() as tmp:
        objs = [os.path.join(tmp, os.path.basename(src) + ".o") for src in SOURCES]
        compiles = [[nvcc_path(), *flags, "-c", "-o", obj, src] for obj, src in zip(objs, SOURCES)] if do_lib else []
        ok, text = _compile_all(compiles + ([ext_command(ext_tmp)] if do_ext else []))
        if ok and do_lib:
            ok, linked = _compile_all([[nvcc_path(), *flags, "-shared", "-o", lib_tmp, *objs]])
            text += linked
    if verbose or not ok:
        sys.stderr.write(text)
    if not ok:
        for path in (lib_tmp, ext_tmp):
            if os.path.exists(path):
                os.remove(path)
        raise RuntimeError("the compiler failed building " + " and ".join(n for n, d in (("libdgemm.so", do_lib), ("_marshal.so", do_ext)) if d))
    if do_lib:
        if check and not extra:
            check_ptxas(text)
        os.replace(lib_tmp, LIB)
    if do_ext:
        os.replace(ext_tmp, EXT)
        with open(EXT_STAMP, "w") as f:
            f.write(version)
    if version is None:
        sys.stderr.write("torch is not installed: libdgemm.so is built, the Python module _marshal is not\n")
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
