"""What the C library's build needs: nvcc.  The binding's compiled part needs torch besides, and comes behind it.  (The compilers are stand-ins that note their command.)"""
import subprocess
import sys

import pytest

from paper_2012_01114_b200 import build


@pytest.fixture
def commands(monkeypatch, tmp_path):
    ran = []

    def run(cmd, **kw):
        ran.append(cmd)
        if cmd[0] in fails:
            raise subprocess.CalledProcessError(1, cmd)
        open(cmd[cmd.index("-o") + 1], "w").close()

    fails = set()
    monkeypatch.setattr(build, "LIB", str(tmp_path / "libpsa.so"))
    monkeypatch.setattr(build, "MARSHAL", str(tmp_path / "psa_marshal.so"))
    monkeypatch.setattr(build.subprocess, "check_call", run)
    return ran, fails, tmp_path


def test_without_torch(commands, monkeypatch, capsys):
    ran, _, path = commands
    monkeypatch.setitem(sys.modules, "torch", None)          # (an import of it fails)
    assert build.build(force=True) == str(path / "libpsa.so") and (path / "libpsa.so").exists()
    assert len(ran) == 1 and "nvcc" in ran[0][0] and "torch" in capsys.readouterr().err


def test_the_library_comes_first(commands):
    ran, fails, path = commands
    fails.add("g++")
    with pytest.raises(subprocess.CalledProcessError):
        build.build(force=True)
    assert (path / "libpsa.so").exists() and not (path / "psa_marshal.so").exists()


def test_both(commands):
    ran, _, path = commands
    build.build()
    assert [c[0].split("/")[-1] for c in ran] == ["nvcc", "g++"] and (path / "psa_marshal.so").exists()
    build.build()                                            # nothing is newer
    assert len(ran) == 2
