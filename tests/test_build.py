"""The build on machines that lack a part of what it uses: stand-ins for the compilers write their output file."""
import os
import stat
import time
import warnings

import pytest

from paper_2608_16305_b200 import build

FAKE = """#!/bin/sh
while [ $# -gt 0 ]; do
  if [ "$1" = "-o" ]; then echo built > "$2"; echo "$0" >> "%s"; fi
  shift
done
"""


@pytest.fixture
def tree(tmp_path, monkeypatch):
    """A package folder of its own with compilers that log each run."""
    (tmp_path / "pkg" / "csrc").mkdir(parents=True)
    (tmp_path / "include").mkdir()
    old = time.time() - 1000
    for f in ("pkg/csrc/a.cu", "pkg/csrc/b.cuh", "pkg/csrc/marshal.c", "include/tgnn.h"):
        (tmp_path / f).write_text("")
        os.utime(tmp_path / f, (old, old))
    log = tmp_path / "runs"
    for name in ("nvcc", "cc"):
        p = tmp_path / name
        p.write_text(FAKE % log)
        p.chmod(p.stat().st_mode | stat.S_IXUSR)
    monkeypatch.setenv("NVCC", str(tmp_path / "nvcc"))
    monkeypatch.setenv("CC", str(tmp_path / "cc"))
    here = str(tmp_path / "pkg")
    monkeypatch.setattr(build, "HERE", here)
    monkeypatch.setattr(build, "CSRC", os.path.join(here, "csrc"))
    monkeypatch.setattr(build, "LIB", os.path.join(here, "lib.so"))
    monkeypatch.setattr(build, "MARSHAL", os.path.join(here, "_marshal.so"))

    def runs():
        names = [os.path.basename(x) for x in log.read_text().split()] if log.exists() else []
        log.write_text("")
        return names
    return tmp_path, runs


def test_both_are_built_once(tree):
    tmp, runs = tree
    assert build.needs_build()
    assert build.build_library() == build.LIB and runs() == ["nvcc", "cc"]
    assert not build.needs_build()
    build.build_library()
    assert runs() == []
    build.build_library(force=True)
    assert runs() == ["nvcc", "cc"]


@pytest.mark.parametrize("cc", ["missing", "/bin/false"])
def test_without_a_c_compiler_the_library_is_there(tree, monkeypatch, cc):
    """A user of the training step needs no argument marshalling: the library is built, and a warning says what cannot be called."""
    tmp, runs = tree
    monkeypatch.setenv("CC", str(tmp / cc) if cc == "missing" else cc)
    with pytest.warns(UserWarning, match="history"):
        assert build.build_library() == build.LIB
    assert os.path.exists(build.LIB) and not os.path.exists(build.MARSHAL) and runs() == ["nvcc"]
    assert not build.needs_build()                                 # the library is up to date
    with pytest.warns(UserWarning, match="history"):
        build.build_library()
    assert runs() == []                                            # and is not compiled again for the missing part
    monkeypatch.setenv("CC", str(tmp / "cc"))
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        build.build_library()
    assert os.path.exists(build.MARSHAL) and runs() == ["cc"]


def test_a_marshalling_module_of_older_sources_does_not_stay(tree, monkeypatch):
    tmp, runs = tree
    build.build_library()
    runs()
    later = time.time() + 1000
    os.utime(tmp / "pkg" / "csrc" / "marshal.c", (later, later))
    monkeypatch.setenv("CC", "/bin/false")
    with pytest.warns(UserWarning, match="history"):
        build.build_library()
    assert not os.path.exists(build.MARSHAL) and runs() == []


@pytest.mark.parametrize("changed,want", [("pkg/csrc/a.cu", ["nvcc"]), ("pkg/csrc/b.cuh", ["nvcc"]), ("pkg/csrc/marshal.c", ["cc"]),
                                          ("include/tgnn.h", ["nvcc", "cc"])])
def test_what_a_change_builds(tree, changed, want):
    tmp, runs = tree
    build.build_library()
    runs()
    later = time.time() + 1000
    os.utime(tmp / changed, (later, later))
    build.build_library()
    assert runs() == want
