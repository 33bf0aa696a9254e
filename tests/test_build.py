"""What is built again after a change: every header that a source includes is among what its age is compared with."""
import os
import re

import pytest

from paper_2303_04769_amd import build


def included(path, seen=None):
    """The repository's own headers that a source takes in, by whatever way."""
    seen = set() if seen is None else seen
    for name in re.findall(r'^\s*#include\s+"([^"]+)"', open(path).read(), re.M):
        at = os.path.realpath(os.path.join(os.path.dirname(path), name))
        assert os.path.exists(at), (path, name)
        if at not in seen:
            seen.add(at)
            included(at, seen)
    return seen


@pytest.fixture
def compared(monkeypatch):
    """What each target's age is compared with, and nothing built."""
    found = {}
    monkeypatch.setattr(build, "_stale", lambda target, deps: found.__setitem__(os.path.basename(target), {os.path.realpath(d) for d in deps}))
    return found


def test_the_extension(compared):
    build.build_fastcall()
    deps = compared[os.path.basename(build.FASTCALL)]
    src = os.path.join(build.CSRC, "fastcall.cpp")
    assert os.path.realpath(src) in deps and included(src) <= deps


def test_the_library(compared, monkeypatch, tmp_path):
    (tmp_path / "flags.txt").write_text(" ".join(build.FLAGS))
    monkeypatch.setattr(build, "OBJ", str(tmp_path))
    build.build_lib()
    for name in build.SOURCES:
        src = os.path.join(build.CSRC, name)
        deps = compared[name.replace(".hip", ".o")]
        assert os.path.realpath(src) in deps and included(src) <= deps, (name, included(src) - deps)
    probe = os.path.join(build.CSRC, "probe.hip")
    assert included(probe) <= compared[os.path.basename(build.PROBE_LIB)]
