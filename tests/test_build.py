"""Building: what it needs, and what the built files refer to."""
import ast
import shutil
import subprocess
import sys

import pytest

from paper_2511_05814_amd import build


def test_the_c_library_needs_no_torch(monkeypatch, capsys):
    monkeypatch.setitem(sys.modules, "torch", None)   # importing it raises ImportError
    monkeypatch.setattr(build.subprocess, "run", lambda *a, **k: 1 / 0)
    assert build.build_ops() is None
    assert "torch is not installed" in capsys.readouterr().err


def test_the_module_takes_the_library_beside_it(tmp_path):
    """In a copy of the tree the module must not load the library of the tree
    that it was built in."""
    pytest.importorskip("torch")
    for path in (build.OUT, build.OPS):
        shutil.copy(path, tmp_path)
    code = """
import importlib.machinery, importlib.util, sys, torch
path = sys.argv[1] + "/_attention_ops.so"
loader = importlib.machinery.ExtensionFileLoader("_attention_ops", path)
loader.exec_module(importlib.util.module_from_spec(importlib.util.spec_from_loader("_attention_ops", loader)))
print({line.split()[-1] for line in open("/proc/self/maps") if "libmoe_offload" in line})
"""
    out = subprocess.run([sys.executable, "-c", code, str(tmp_path)], capture_output=True, text=True, check=True).stdout
    assert ast.literal_eval(out) == {str(tmp_path / "libmoe_offload.so")}
