"""The C library is built whatever becomes of the 8-bit layers' Python module, which needs torch's headers and another compiler.
No compiler runs here: commands are looked at and answered."""
import subprocess
import types

import pytest

from paper_2307_16273_amd import build


@pytest.fixture
def commands(monkeypatch, tmp_path):
    """Every command that the build would have run; g++ fails where `fails` says so."""
    ran = []

    def answer(cmd, **kw):
        ran.append(cmd)
        return types.SimpleNamespace(returncode=int(cmd[0] == "g++" and answer.fails), stdout="", stderr="")

    answer.fails = False
    monkeypatch.setattr(build, "HERE", str(tmp_path))
    monkeypatch.setattr(build, "MODULE", str(tmp_path / "_layers8.so"))
    monkeypatch.setattr(build, "OUT", str(tmp_path / "libzkdl.so"))
    monkeypatch.setattr(subprocess, "run", answer)
    return ran, answer


def linked(ran):
    return [c for c in ran if "-shared" in c and c[0] == "hipcc"]


def test_library_is_linked_where_the_module_fails(commands, capsys):
    ran, answer = commands
    answer.fails = True
    with pytest.raises(RuntimeError, match="layers8_torch"):
        build.build(verbose=False)
    assert len(linked(ran)) == 1


def test_library_is_built_without_what_the_module_needs(commands, capsys, monkeypatch):
    import shutil
    ran, _ = commands
    monkeypatch.setattr(shutil, "which", lambda name, *a, **k: None)
    stale = build.MODULE
    open(stale, "w").close()
    assert build.build(verbose=False) == build.OUT
    assert len(linked(ran)) == 1 and not [c for c in ran if c[0] == "g++"]
    assert "8-bit layers" in capsys.readouterr().err
    with pytest.raises(FileNotFoundError):       # a module of an older source does not stay in its place
        open(stale)


def test_library_is_built_without_torchs_headers(commands, capsys, monkeypatch, tmp_path):
    from torch.utils import cpp_extension
    ran, _ = commands
    monkeypatch.setattr(cpp_extension, "include_paths", lambda *a, **k: [str(tmp_path)])
    assert build.build(verbose=False) == build.OUT
    assert len(linked(ran)) == 1 and not [c for c in ran if c[0] == "g++"]
    assert "python_variable.h" in capsys.readouterr().err
