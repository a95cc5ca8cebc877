"""The build of the library does not need what only its extension for torch does."""
import importlib.util
import shutil
import subprocess

import pytest


@pytest.fixture
def build(monkeypatch, tmp_path):
    from paper_2510_23264_amd import build as b
    commands = []
    monkeypatch.setattr(b, "HERE", str(tmp_path))
    monkeypatch.setattr(b, "LIB", str(tmp_path / "libpahq.so"))
    monkeypatch.setattr(b, "EXTENSION", str(tmp_path / "_tensors.so"))
    monkeypatch.setattr(subprocess, "run", lambda command, **how: commands.append(command))
    (tmp_path / "_tensors.so").write_bytes(b"of before")
    return b, commands, tmp_path


def test_the_library_and_its_extension(build):
    b, commands, _ = build
    assert b.build() == b.LIB
    assert [c[0] for c in commands] == ["hipcc"] * (len(b.SOURCES) + 1) + ["g++"]
    assert b.LIB in commands[-2] and b.EXTENSION in commands[-1]


@pytest.mark.parametrize("missing", ["torch", "g++"])
def test_the_library_alone(build, monkeypatch, missing):
    b, commands, path = build
    find, which = importlib.util.find_spec, shutil.which
    if missing == "torch":
        monkeypatch.setattr(importlib.util, "find_spec", lambda name, *a: None if name == "torch" else find(name, *a))
    else:
        monkeypatch.setattr(shutil, "which", lambda name, *a, **k: None if name == "g++" else which(name, *a, **k))
    with pytest.warns(UserWarning, match=missing.replace("+", r"\+")):
        assert b.build() == b.LIB
    assert [c[0] for c in commands] == ["hipcc"] * (len(b.SOURCES) + 1) and b.LIB in commands[-1]
    assert not (path / "_tensors.so").exists()


def test_an_extension_that_does_not_compile_is_an_error(build, monkeypatch):
    b, commands, _ = build

    def run(command, **how):
        if command[0] == "g++":
            raise subprocess.CalledProcessError(1, command)
    monkeypatch.setattr(subprocess, "run", run)
    with pytest.raises(subprocess.CalledProcessError):
        b.build()
