"""The quick calls from Python are an extra: a machine that cannot compile them still gets the library, and no stale or half-written module."""
import os
import stat

import pytest

from paper_1611_08035_b200 import build


def compiler(folder, text):
    """A g++ of that text, first in the path."""
    folder.mkdir()
    f = folder / "g++"
    f.write_text("#!/bin/sh\n" + text)
    f.chmod(f.stat().st_mode | stat.S_IXUSR)
    return str(folder)


@pytest.fixture
def elsewhere(monkeypatch, tmp_path):
    build.build()  # the library itself is there
    monkeypatch.setattr(build, "CALLS_PATH", tmp_path / "_b2calls.so")
    monkeypatch.setattr(build, "CALLS_STAMP", tmp_path / "calls.stamp", raising=False)
    return tmp_path


def test_library_builds_without_the_quick_calls(elsewhere, monkeypatch, capsys):
    build.CALLS_PATH.write_text("of an earlier build")
    monkeypatch.setenv("PATH", compiler(elsewhere / "bin", "echo no such header >&2; exit 1\n") + os.pathsep + os.environ["PATH"])
    assert build.build() == build.LIB_PATH
    assert not build.CALLS_PATH.exists(), "a module that does not belong to this library's sources would be loaded"
    assert "no such header" in capsys.readouterr().err


def test_no_compiler_at_all(elsewhere, monkeypatch):
    monkeypatch.setenv("PATH", str(elsewhere / "nothing here"))
    assert build.build() == build.LIB_PATH and not build.CALLS_PATH.exists()


def test_the_module_appears_whole(elsewhere, monkeypatch):
    """The compiler writes to another name; what is importable is replaced at once, and not compiled again without need."""
    monkeypatch.setenv("PATH", compiler(elsewhere / "bin", f'''echo run >> {elsewhere}/runs
while [ "$1" != "-o" ]; do shift; done
[ "$2" != "{build.CALLS_PATH}" ] || exit 1
echo compiled > "$2"\n''') + os.pathsep + os.environ["PATH"])
    build.build()
    build.build()
    assert build.CALLS_PATH.read_text() == "compiled\n" and (elsewhere / "runs").read_text() == "run\n"
    assert sorted(f.name for f in elsewhere.iterdir()) == ["_b2calls.so", "bin", "calls.stamp", "runs"]
