"""Which objects an incremental build compiles again (on empty files of the same names; no compiler runs)."""
import os
import re

import pytest

from paper_2512_21571_amd import _build

INCLUDE = re.compile(r'#include "([^"]+)"')


def included():
    """Every header of this repository that the sources include, directly or through one another."""
    todo, seen = [os.path.join(_build.CSRC, s) for s in _build.SOURCES], set()
    while todo:
        path = todo.pop()
        for name in INCLUDE.findall(open(path).read()):
            h = os.path.normpath(os.path.join(os.path.dirname(path), name))
            if os.path.exists(h) and h not in seen:
                seen.add(h)
                todo.append(h)
    return sorted(seen)


@pytest.mark.parametrize("header", [os.path.relpath(h, _build.HERE) for h in included()])
def test_a_changed_header_rebuilds_every_object(header, tmp_path, monkeypatch):
    here = tmp_path / "package"
    csrc, obj = here / "csrc", here / "_build"
    csrc.mkdir(parents=True), obj.mkdir(), (tmp_path / "include").mkdir()
    files = [csrc / s for s in _build.SOURCES] + [here / os.path.relpath(h, _build.HERE) for h in included()]
    for f in files:
        f.touch()
        os.utime(f, (1000, 1000))
    for f in [obj / (s + ".o") for s in _build.SOURCES] + [here / "libnnc.so"]:
        f.touch()
        os.utime(f, (2000, 2000))
    ran = []
    for name, value in dict(HERE=str(here), CSRC=str(csrc), OBJ_DIR=str(obj), LIB_PATH=str(here / "libnnc.so"), _run=ran.append).items():
        monkeypatch.setattr(_build, name, value)
    _build.build(force=False)
    assert not ran and not _build.is_stale()
    os.utime(here / header, (3000, 3000))
    assert _build.is_stale()
    _build.build(force=False)
    assert sorted(c[-1] for c in ran[:-1]) == sorted(str(csrc / s) for s in _build.SOURCES) and "-shared" in ran[-1]
