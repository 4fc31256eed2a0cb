"""Integers that 32 bits do not hold are refused by the Python functions, not cut to their low bits (no GPU)."""

import os

import pytest

import paper_2510_08726_amd as pa


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(pa.library_path()):
        import __graft_entry__
        __graft_entry__.build()
    return pa.load_library()


BIG = 1 << 32


def test_sizes_that_are_not_supported():
    assert pa.kv4_page_bytes(BIG + 64, 128) == 0 and pa.kv4_page_bytes(64, BIG + 128) == 0
    assert pa.kv4_page_bytes(64 - BIG, 128) == 0
    for bad in ((BIG + 1, 8, 2, 128), (1, BIG + 8, 2, 128), (1, 8, BIG + 2, 128), (1, 8, 2, BIG + 128)):
        assert pa.attn_decode_kv4_workspace_bytes(*bad) == 0


def test_frequencies(monkeypatch):
    # (nothing is allocated for them)
    monkeypatch.setattr(pa.torch, "empty", lambda *a, **k: pytest.fail("allocated"))
    for n in (BIG + 64, 64 - BIG, 1 << 31):
        with pytest.raises((ValueError, pa.AttnError)):
            pa.rope_frequencies(n)
