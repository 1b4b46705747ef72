"""What the package and its build need of a machine (no GPU needed)."""

import os
import shutil
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def python(code):
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stdout + r.stderr
    return r.stdout


def test_all_names_without_torch():
    python("import sys; sys.modules['torch'] = None\n"
           "from paper_2607_01408_amd import *\n"
           "Plan, paths_host\n")


def test_the_operators_are_listed_and_found():
    python("import paper_2607_01408_amd as sg\n"
           "assert {'rms_norm', 'gated', 'Block8', 'Plan'} <= set(dir(sg))\n"
           "assert callable(sg.rms_norm)\n")


@pytest.fixture
def small(monkeypatch, tmp_path):
    """build.py with one source and everything it writes under tmp_path."""
    from paper_2607_01408_amd import build

    os.symlink(os.path.join(ROOT, "include"), tmp_path / "include")
    monkeypatch.setattr(build, "ROOT", str(tmp_path))
    monkeypatch.setattr(build, "SOURCES", ["feedforward.cpp"])
    monkeypatch.setattr(build, "LIB", str(tmp_path / "lib.so"))
    monkeypatch.setattr(build, "BINDING", str(tmp_path / "binding.so"))
    return build


def test_the_library_is_built_without_torch(small, monkeypatch, capsys):
    monkeypatch.setitem(sys.modules, "torch", None)
    small.build()
    assert os.path.exists(small.LIB) and not os.path.exists(small.BINDING)
    assert "not built" in capsys.readouterr().out


def test_the_library_is_built_where_the_binding_is_not(small, monkeypatch):
    monkeypatch.setattr(small, "binding_command", lambda out: ["false"])
    with pytest.raises(RuntimeError, match="binding.cpp"):
        small.build()
    assert os.path.exists(small.LIB) and not os.path.exists(small.BINDING)


def test_the_binding_needs_no_other_compiler(small, monkeypatch):
    which = shutil.which
    monkeypatch.setattr(shutil, "which", lambda name, *a, **k: None if name in ("g++", "c++") else which(name, *a, **k))
    assert os.path.exists(small.binding_command("x.so")[0])
