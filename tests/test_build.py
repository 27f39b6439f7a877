"""Building: what it needs, and what the built files refer to."""
import sys

from paper_2511_05814_amd import build


def test_the_c_library_needs_no_torch(monkeypatch, capsys):
    monkeypatch.setitem(sys.modules, "torch", None)   # importing it raises ImportError
    monkeypatch.setattr(build.subprocess, "run", lambda *a, **k: 1 / 0)
    assert build.build_ops() is None
    assert "torch is not installed" in capsys.readouterr().err
