"""The build compiles again what a change of its flags concerns, and nothing else (a stand-in for nvcc notes its command lines)."""
import importlib.util
import os
import shutil
import stat

import pytest

from paper_2009_02701_b200 import build as real

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture
def tree(tmp_path, monkeypatch):
    """A copy of the sources with a stand-in for nvcc; returns its package, run(), which imports and runs the copy's build and gives the
    command lines, and age()."""
    package = tmp_path / "paper_2009_02701_b200"
    package.mkdir()
    shutil.copytree(real.CSRC, package / "csrc")
    shutil.copytree(os.path.join(ROOT, "include"), tmp_path / "include")
    shutil.copy2(real.__file__, package / "build.py")
    log, fake = tmp_path / "log", tmp_path / "nvcc"
    fake.write_text('#!/bin/sh\necho "$*" >> %s\nwhile [ "$1" != -o ]; do shift; done\n: > "$2"\n' % log)
    fake.chmod(fake.stat().st_mode | stat.S_IXUSR)
    monkeypatch.setenv("NVCC", str(fake))

    def age(when):
        """The clock of file times is coarse: what exists is made old, so that what comes later is newer."""
        for folder, _, files in os.walk(tmp_path):
            for f in files:
                path = os.path.join(folder, f)
                if os.path.getmtime(path) > when:
                    os.utime(path, (when, when))

    age(1_000_000_000)

    def run(**kw):
        spec = importlib.util.spec_from_file_location("copied_build", package / "build.py")
        module = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(module)
        log.write_text("")
        module.build(**kw)
        return log.read_text().splitlines()

    return package, run, age


def test_a_change_of_flags_compiles_everything_again(tree):
    package, run, age = tree
    units = len(real.SOURCES)
    first = run()
    assert len(first) == units + 1 and all("-O3" in c for c in first)
    assert run() == []
    age(1_100_000_000)
    text = (package / "build.py").read_text()
    (package / "build.py").write_text(text.replace('"-O3"', '"-O2"'))
    again = run()
    assert len(again) == units + 1 and all("-O2" in c for c in again)
    assert run() == []


def test_a_change_of_one_source_compiles_that_one(tree):
    package, run, age = tree
    run()
    age(1_100_000_000)
    os.utime(package / "csrc" / "hpsgd_gemm.cu")
    commands = run()
    assert len(commands) == 2 and "hpsgd_gemm.cu" in commands[0] and "-shared" in commands[1]
