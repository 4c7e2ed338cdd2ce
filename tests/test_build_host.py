"""What a build runs, with nothing run: the library needs ROCm's compiler alone, and the binding
is built where torch is."""
import os
import shutil
import subprocess
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


def test_a_moved_package_uses_its_own_library(tmp_path):
    """Not the one at the place where it was built."""
    pytest.importorskip("torch")
    if not os.path.exists(build.BINDING):
        build.build()
    package = os.path.basename(build.HERE)
    there = tmp_path / package
    there.mkdir()
    for name in os.listdir(build.HERE):
        if name.endswith((".py", ".so")):
            shutil.copy(os.path.join(build.HERE, name), there / name)
    code = (f"import {package} as p; p.lib(); p.sequence._binding()\n"
            "print(*{l.split()[-1] for l in open('/proc/self/maps') if 'libadst' in l})")
    r = subprocess.run([sys.executable, "-c", code], cwd=tmp_path, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    assert r.stdout.split() == [str(there / "libadst.so")]
