"""What a build runs, with nothing run: the library needs ROCm's compiler alone, and the binding
is built where torch is."""
import os
import sys

import pytest

from paper_2509_02197_amd import build


@pytest.fixture
def commands(monkeypatch, tmp_path):
    ran = []
    monkeypatch.setattr(build, "BUILD", str(tmp_path))
    monkeypatch.setattr(build, "_run", lambda cmd, verbose: ran.append(cmd))
    monkeypatch.setattr(build.os, "replace", lambda a, b: ran.append(["replace", a, b]))
    return ran


def names(commands):
    return {os.path.basename(c) for cmd in commands for c in cmd}


def test_the_library_without_torch(commands, monkeypatch):
    monkeypatch.setitem(sys.modules, "torch", None)  # import torch raises ImportError
    assert build.build() == build.LIB
    assert {"recurrence.hip", "abi.cpp", "libadst.so"} <= names(commands)
    assert not {"binding.cpp", "_binding.so"} & names(commands)
    assert {os.path.basename(c[0]) for c in commands} == {"hipcc", "replace"}


def test_the_library_is_there_before_the_binding_can_fail(commands, monkeypatch):
    pytest.importorskip("torch")

    def run(cmd, verbose):
        if any("binding" in c for c in cmd):
            raise RuntimeError("compile failed")
        commands.append(cmd)

    monkeypatch.setattr(build, "_run", run)
    with pytest.raises(RuntimeError):
        build.build()
    assert commands[-1] == ["replace", build.LIB + ".tmp", build.LIB]


def test_library_and_binding(commands):
    pytest.importorskip("torch")
    build.build()
    assert commands[-1] == ["replace", build.BINDING + ".tmp", build.BINDING]
    assert {os.path.basename(c[0]) for c in commands} == {"hipcc", "replace"}
