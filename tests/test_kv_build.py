"""The build on hosts where the key/value cache's binding cannot be built: the store's
library and binding are built all the same (CPU only; nothing is compiled here)."""
import importlib.util
import os
import subprocess

import pytest

from paper_2607_26566_gb300 import build as b


class Done:
    returncode, stdout = 0, ""

    def communicate(self):
        return "", None


@pytest.fixture
def ran(monkeypatch):
    """The commands that a build would run; they all succeed."""
    commands = []

    def run(cmd, *a, **k):
        commands.append(cmd)
        return Done()

    monkeypatch.setattr(subprocess, "run", run)
    monkeypatch.setattr(subprocess, "Popen", run)
    monkeypatch.setattr(os, "replace", lambda *a: None)
    return commands


def built(commands):
    return {name for name in (b.PYCALL, b.KVCALL, b.LIB) for c in commands if name + ".tmp" in c}


def test_all_of_it_where_torch_has_cuda(ran, capfd):
    assert b.build() == b.LIB
    assert built(ran) == {b.LIB, b.PYCALL, b.KVCALL}
    assert capfd.readouterr().err == ""


def test_without_torch(ran, capfd, monkeypatch):
    find = importlib.util.find_spec
    monkeypatch.setattr(importlib.util, "find_spec", lambda name, *a: None if name == "torch" else find(name, *a))
    assert b.build() == b.LIB
    assert built(ran) == {b.LIB, b.PYCALL}
    assert "KVCache" in capfd.readouterr().err
    with pytest.raises(RuntimeError, match="torch"):
        b.build_kvcall()


def test_with_a_torch_without_cuda(ran, capfd, monkeypatch, tmp_path):
    (tmp_path / "lib").mkdir()
    (tmp_path / "lib" / "libc10.so").touch()
    (tmp_path / "__init__.py").touch()
    spec = importlib.util.spec_from_file_location("torch", tmp_path / "__init__.py")
    find = importlib.util.find_spec
    monkeypatch.setattr(importlib.util, "find_spec", lambda name, *a: spec if name == "torch" else find(name, *a))
    assert b.build() == b.LIB
    assert built(ran) == {b.LIB, b.PYCALL}
    assert "KVCache" in capfd.readouterr().err


def test_a_build_without_the_binding_is_not_stale_for_that(monkeypatch, tmp_path):
    for name in ("LIB", "PYCALL", "KVCALL"):
        monkeypatch.setattr(b, name, str(tmp_path / name))
    monkeypatch.setattr(b, "_inputs", lambda: [])
    for name in ("LIB", "PYCALL"):
        (tmp_path / name).touch()
    assert b.is_stale()
    find = importlib.util.find_spec
    monkeypatch.setattr(importlib.util, "find_spec", lambda name, *a: None if name == "torch" else find(name, *a))
    assert not b.is_stale()


def test_a_failing_compilation_is_still_an_error(ran, monkeypatch):
    class Failed(Done):
        returncode = 1

    monkeypatch.setattr(subprocess, "run", lambda cmd, *a, **k: Failed() if b.KVCALL + ".tmp" in cmd else Done())
    with pytest.raises(RuntimeError, match="binding build failed"):
        b.build()
