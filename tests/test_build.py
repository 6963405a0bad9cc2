"""The build without torch and after a change of torch, on a stand-in for the library's sources. No GPU."""
import os
import subprocess
import sys

import pytest

from paper_2003_00532_b200 import build as _build


@pytest.fixture
def small(tmp_path, monkeypatch):
    """A library of one small source; the module's compile is replaced by a copy that is counted."""
    src = tmp_path / "one.cu"
    src.write_text('extern "C" int one() { return 1; }\n')
    monkeypatch.setattr(_build, "SOURCES", [str(src)])
    monkeypatch.setattr(_build, "LIB", str(tmp_path / "lib.so"))
    monkeypatch.setattr(_build, "EXT", str(tmp_path / "ext.so"))
    monkeypatch.setattr(_build, "EXT_STAMP", str(tmp_path / "ext.so.torch"), raising=False)
    monkeypatch.setenv("DGEMM_NVCC_FLAGS", "-O0")
    return tmp_path


def _count_ext(monkeypatch):
    calls = []

    def command(out):
        calls.append(out)
        return ["cp", _build.EXT_SOURCE, out]

    monkeypatch.setattr(_build, "ext_command", command)
    return calls


def test_the_library_is_built_without_torch(small, monkeypatch, capsys):
    monkeypatch.setitem(sys.modules, "torch", None)          # `import torch` raises ImportError
    assert _build.build() == str(small / "lib.so")
    assert os.path.exists(small / "lib.so") and not os.path.exists(small / "ext.so")
    assert "torch is not installed" in capsys.readouterr().err
    assert not _build.is_stale()
    monkeypatch.delitem(sys.modules, "torch")
    assert _build.is_stale()                                  # with torch the module is missing


def test_another_torch_makes_the_module_stale_and_the_library_not(small, monkeypatch):
    calls = _count_ext(monkeypatch)
    _build.build()
    assert len(calls) == 1 and not _build.is_stale()
    _build.build()
    assert len(calls) == 1
    built = os.path.getmtime(small / "lib.so")
    monkeypatch.setattr(_build, "torch_version", lambda: "torch 99.0, 3.99")
    assert _build.is_stale()
    _build.build()
    assert len(calls) == 2 and os.path.getmtime(small / "lib.so") == built and not _build.is_stale()


def test_a_failed_compile_leaves_nothing_behind(small, monkeypatch):
    monkeypatch.setattr(_build, "ext_command", lambda out: ["false"])
    with pytest.raises(RuntimeError):
        _build.build()
    assert sorted(os.listdir(small)) == ["one.cu"]


def test_a_missing_module_is_named():
    program = ("import paper_2003_00532_b200 as dg, os\n"
               "from paper_2003_00532_b200 import binding\n"
               "binding._HERE = '/nonexistent'\n"
               "lib = binding.load_library()\n"
               "try:\n    dg.layernorm_fwd\n"
               "except FileNotFoundError as e:\n    assert '_marshal.so' in str(e)\n    print('named')\n")
    _build.build()
    run = subprocess.run([sys.executable, "-c", program], capture_output=True, text=True,
                         cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    assert run.stdout == "named\n", run.stdout + run.stderr
