"""The build without a compiler's work: the C library is linked whatever becomes of the Python module beside it."""
import subprocess

import pytest

from paper_2508_17588_amd import build as B


def test_library_is_linked_where_the_python_module_cannot_be_compiled(monkeypatch, tmp_path):
    commands = []

    def run(cmd, **_):
        commands.append(cmd)
        module = any(str(c).endswith("fp8_binding.cpp") for c in cmd)
        return subprocess.CompletedProcess(cmd, 1 if module else 0, "", "no such header" if module else "")
    monkeypatch.setattr(B.subprocess, "run", run)
    monkeypatch.setattr(B, "BUILD_DIR", str(tmp_path))
    with pytest.raises(RuntimeError, match="fp8_binding"):
        B.build(verbose=False)
    assert any(B.LIB_PATH in cmd and "-shared" in cmd for cmd in commands), "not linked"


def test_library_is_linked_without_torch(monkeypatch, tmp_path):
    commands = []
    monkeypatch.setattr(B.subprocess, "run", lambda cmd, **_: commands.append(cmd) or subprocess.CompletedProcess(cmd, 0, "", ""))
    monkeypatch.setattr(B, "BUILD_DIR", str(tmp_path))

    def missing():
        raise ImportError("No module named 'torch'")
    monkeypatch.setattr(B, "_build_binding", missing)
    with pytest.raises(ImportError, match="torch"):
        B.build(verbose=False)
    assert any(B.LIB_PATH in cmd and "-shared" in cmd for cmd in commands), "not linked"
