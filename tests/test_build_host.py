"""What the build needs: hipcc, and for the Python module torch (no GPU, and nothing is compiled here)."""

import subprocess
import sys
from types import SimpleNamespace

import pytest

from paper_2511_01385_amd import build


@pytest.fixture
def commands(monkeypatch):
    """The commands that a build would run, every one of them a success."""
    ran = []
    monkeypatch.setattr(subprocess, "run", lambda cmd, **kw: ran.append(cmd) or SimpleNamespace(returncode=0, stderr=""))
    monkeypatch.setattr(build.shutil, "move", lambda *a: None)
    monkeypatch.setattr(build.os, "makedirs", lambda *a, **kw: None)
    monkeypatch.setattr(build, "HIPCC", sys.executable)  # (a file that exists)
    return ran


def test_no_compiler_but_hipcc(commands, monkeypatch):
    monkeypatch.setenv("CXX", "/nonexistent/c++")
    assert build.build(verbose=False) == build.LIB
    assert len(commands) == len(build.SOURCES) + 2
    assert {c[0] for c in commands} == {sys.executable}


def test_without_torch_the_library_alone(commands, monkeypatch):
    monkeypatch.setitem(sys.modules, "torch", None)  # (an import of it fails)
    assert build.build(verbose=False) == build.LIB
    assert len(commands) == len(build.SOURCES) + 1
