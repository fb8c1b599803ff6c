"""What building the package needs, with the compilers' calls recorded in place of made."""
import importlib.util
import subprocess
from pathlib import Path

import pytest

from paper_2504_18454_b200 import build


@pytest.fixture
def calls(monkeypatch, tmp_path):
    """The outputs of the compiler calls, in order; the built files lie in a folder of their own."""
    made = []

    def call(cmd, **kw):
        out = Path(cmd[cmd.index("-o") + 1])
        out.write_bytes(b"")
        made.append(out.name.split(".")[0])

    monkeypatch.setattr(build, "HERE", tmp_path / "package")
    (tmp_path / "package").mkdir(), (tmp_path / "include").mkdir()
    monkeypatch.setattr(build, "LIB", tmp_path / "package" / "libpalsgd.so")
    monkeypatch.setattr(build, "EXT", tmp_path / "package" / "_block.so")
    for h in ("palsgd.h", "palsgd_block.h"):
        (tmp_path / "include" / h).write_text("")
    monkeypatch.setattr(subprocess, "check_call", call)
    return made


def test_both_are_built_where_torch_is_there(calls):
    build.build(force=True)
    assert sorted(calls) == ["_block", "libpalsgd"]
    build.build()
    assert len(calls) == 2                               # up to date


def test_the_library_is_built_without_torch(calls, monkeypatch, capsys):
    find = importlib.util.find_spec
    monkeypatch.setattr(importlib.util, "find_spec", lambda name, *a: None if name == "torch" else find(name, *a))
    monkeypatch.setitem(__import__("sys").modules, "torch", None)
    assert build.build(force=True) == build.LIB and calls == ["libpalsgd"]
    assert "_block.so" in capsys.readouterr().err


def test_a_binding_that_does_not_compile_leaves_the_library_built(calls, monkeypatch):
    call = subprocess.check_call

    def no_headers(cmd, **kw):
        if "_block" in str(cmd[cmd.index("-o") + 1]):
            raise subprocess.CalledProcessError(1, cmd)
        call(cmd, **kw)

    monkeypatch.setattr(subprocess, "check_call", no_headers)
    with pytest.raises(subprocess.CalledProcessError):
        build.build(force=True)
    assert calls == ["libpalsgd"] and build.LIB.exists()
