"""The library builds where torch or a host compiler is missing: only the binding's host module needs them, and the binding goes without it."""
import subprocess
import sys

import pytest

from paper_2302_06361_amd import build


@pytest.fixture
def linked(monkeypatch, tmp_path):
    """build() with nothing to compile; the commands it runs are kept, not run"""
    commands = []
    monkeypatch.setattr(build, "UNITS", [])
    monkeypatch.setattr(build, "bundle_so", lambda: str(tmp_path / "module.so"))
    monkeypatch.setattr(subprocess, "check_call", lambda command, *a, **k: commands.append(command))
    return commands


def test_without_torch(linked, monkeypatch, capsys):
    monkeypatch.setitem(sys.modules, "torch", None)         # (an import of it fails)
    for force in (False, True):
        assert build.build(force=force) == build.SO
    assert len(linked) == 2 and all(build.SO in c for c in linked)
    assert "host module" in capsys.readouterr().out


def test_without_a_host_compiler(linked, monkeypatch, capsys):
    def check_call(command, *a, **k):
        linked.append(command)
        if command[0] == "g++":
            raise FileNotFoundError(2, "No such file or directory", "g++")
    monkeypatch.setattr(subprocess, "check_call", check_call)
    assert build.build(force=False) == build.SO
    assert "host module" in capsys.readouterr().out


def test_a_module_that_does_not_compile_is_an_error(linked, monkeypatch):
    def check_call(command, *a, **k):
        if command[0] == "g++":
            raise subprocess.CalledProcessError(1, command)
    monkeypatch.setattr(subprocess, "check_call", check_call)
    with pytest.raises(subprocess.CalledProcessError):
        build.build(force=False)
