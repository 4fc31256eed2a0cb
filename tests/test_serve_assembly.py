"""The guards of test_serve_codegen.py read the assembly of the present sources (no GPU)."""

import os
import re

import pytest

from paper_2510_08726_amd import build as libbuild


def _files(tmp_path, monkeypatch):
    monkeypatch.setattr(libbuild, "OBJDIR", str(tmp_path / "obj"))
    monkeypatch.setattr(libbuild, "CSRC", str(tmp_path))
    monkeypatch.setattr(libbuild, "__file__", str(tmp_path / "build.py"))
    sources = [str(tmp_path / n) for n in [*libbuild.SERVE_SOURCES, "build.py"]]
    for f in sources + libbuild.serve_asm_files():
        os.makedirs(os.path.dirname(f), exist_ok=True)
        open(f, "w").close()
    for f in sources:
        os.utime(f, (1000, 1000))
    for f in libbuild.serve_asm_files():
        os.utime(f, (2000, 2000))
    return sources


def test_assembly_older_than_a_source_is_stale(tmp_path, monkeypatch):
    sources = _files(tmp_path, monkeypatch)
    assert not libbuild.serve_asm_stale()
    for f in sources:
        os.utime(f, (3000, 3000))
        assert libbuild.serve_asm_stale(), f
        os.utime(f, (1000, 1000))
    for f in libbuild.serve_asm_files():
        os.utime(f, (500, 500))
        assert libbuild.serve_asm_stale(), f
        os.remove(f)
        assert libbuild.serve_asm_stale(), f
        open(f, "w").close()
        os.utime(f, (2000, 2000))


def test_every_source_counts():
    """What the three units include of this folder, and what that includes."""
    seen, todo = set(), ["rope.hip", "kv4.hip", "decode_kv4.hip"]
    while todo:
        n = todo.pop()
        if n not in seen:
            seen.add(n)
            todo += re.findall(r'^#include "([^"/]+)"', open(os.path.join(libbuild.CSRC, n)).read(), flags=re.M)
    assert seen == set(libbuild.SERVE_SOURCES)


@pytest.mark.parametrize("stale", [False, True])
def test_the_guards_build_where_it_is_stale(monkeypatch, stale):
    import __graft_entry__
    import conftest
    built = []
    monkeypatch.setattr(libbuild, "serve_asm_stale", lambda: stale)
    monkeypatch.setattr(__graft_entry__, "build", lambda: built.append(1))
    conftest.build_where_the_serving_assembly_is_stale()
    assert len(built) == stale
