"""What build_library compiles, and after a change to which files it compiles again (no compiler is started)."""
import os
import re

import pytest

from paper_1906_03707_amd import build


def included(path, seen):
    """The repository's own files that `path` includes, directly or through others."""
    for name in re.findall(r'^\s*#\s*include\s+"([^"]+)"', open(path).read(), re.M):
        for where in (os.path.dirname(path), os.path.join(build.ROOT, "include")):
            full = os.path.normpath(os.path.join(where, name))
            if os.path.exists(full) and full not in seen:
                seen.add(full)
                included(full, seen)
    return seen


def test_every_included_file_is_known():
    seen = set()
    for src in build.SOURCES:
        included(src, seen)
    assert seen and seen <= set(build.SOURCES) | set(build.HEADERS)


def test_every_source_is_compiled():
    csrc = os.path.join(build.HERE, "csrc")
    assert {os.path.join(csrc, f) for f in os.listdir(csrc) if f.endswith((".hip", ".cpp"))} == set(build.SOURCES)


@pytest.mark.parametrize("path", sorted({p for s in build.SOURCES for p in included(s, set())} | set(build.SOURCES)), ids=os.path.basename)
def test_a_change_makes_the_library_old(path, tmp_path, monkeypatch):
    lib = tmp_path / "libhag.so"
    lib.write_bytes(b"")
    monkeypatch.setattr(build, "LIB", str(lib))
    times = {p: os.path.getmtime(p) for p in build.SOURCES + build.HEADERS + [path]}
    newest = max(times.values())
    real = os.path.getmtime
    monkeypatch.setattr(build.os.path, "getmtime", lambda p: newest + 1 if p == str(lib) else newest + 2 if changed and p == path else real(p))
    changed = False
    assert build.build_library(force=False) == str(lib)

    class Started(Exception):
        pass

    def popen(*args, **kwargs):
        raise Started

    monkeypatch.setattr(build.subprocess, "Popen", popen)
    changed = True
    with pytest.raises(Started):
        build.build_library(force=False)
