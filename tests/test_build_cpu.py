"""What a build compiles, and what it needs for that (the commands are recorded, not run)."""
import sys

import pytest

from paper_2607_11985_amd import build


@pytest.fixture
def commands(monkeypatch):
    said = []
    monkeypatch.setattr(build, "_run", lambda cmd, verbose: said.append(cmd))
    monkeypatch.setattr(build, "_run_all", lambda cmds, verbose: said.extend(cmds))
    monkeypatch.setattr(build.os, "replace", lambda a, b: None)
    monkeypatch.setattr(build, "write_embedded_headers", lambda: "jit_headers.cpp")
    return said


def test_the_library_needs_no_torch(commands, monkeypatch):
    monkeypatch.setitem(sys.modules, "torch", None)  # its import raises ImportError
    assert build.build_all(torch_extension=False) == [build.LIB]
    assert all(cmd[0] == build.HIPCC for cmd in commands)
    text = " ".join(word for cmd in commands for word in cmd)
    assert "torch" not in text
    assert all(src in text for src in build.SOURCES)
    with pytest.raises(ImportError):  # asked for, it is not left out without a word
        build.build_all()


def test_the_extension_is_linked_to_the_library(commands):
    assert build.build_all() == [build.LIB, build.TORCH_EXT]
    compiled = [cmd for cmd in commands if cmd[0] == build.CXX]
    assert len(compiled) == 2 and commands[-1] is compiled[-1]
    assert compiled[0][-3].endswith("torch_layers.cpp")
    assert "-l:libvqc.so" in compiled[1] and "-Wl,-rpath,$ORIGIN" in compiled[1]
