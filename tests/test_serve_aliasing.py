"""What the operators around the 4-bit cache write must lie apart from what they read (no GPU).

The C entry points get addresses that are never dereferenced: every call here is refused
before anything is enqueued.
"""

import ctypes
import os

import pytest

import paper_2510_08726_amd as pa

AT = 1 << 20          # spacing of the addresses, more than any operand here takes
D, PAGE = 64, 16
BLOCK = PAGE * D * 17 // 16


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(pa.library_path()):
        import __graft_entry__
        __graft_entry__.build()
    return pa.load_library()


def _ptr(x):
    return ctypes.c_void_p(x)


def _strides(*s):
    return (ctypes.c_longlong * 3)(*s)


B, H, L, PAGES, M = 2, 3, 5, 4, 2
CACHE = PAGES * H * BLOCK
ROWS = B * H * L * D * 2              # bytes of K, V


def load(lib, **at):
    a = dict(cache=1 * AT, table=2 * AT, starts=3 * AT, lens=4 * AT, k=5 * AT, v=6 * AT) | at
    return lib.kv4_load(_ptr(a["cache"]), _ptr(a["table"]), _ptr(a["starts"]), _ptr(a["lens"]), _ptr(a["k"]),
                        _ptr(a["v"]), B, H, L, D, PAGES, PAGE, M, 0, None)


@pytest.mark.parametrize("at", [
    dict(v=5 * AT), dict(v=5 * AT + ROWS - 16), dict(v=5 * AT - ROWS + 16), dict(k=1 * AT), dict(v=1 * AT + CACHE - 16),
    dict(k=1 * AT - ROWS + 16), dict(table=5 * AT + ROWS - 4), dict(starts=6 * AT), dict(lens=6 * AT + 16),
    dict(table=6 * AT - 4 * B * M + 4), dict(lens=5 * AT - 4),
], ids=str)
def test_load(lib, at):
    assert load(lib, **at) == pa.ATTN_ERR_SHAPE


def append(lib, ks=(H * L * D, L * D, D), vs=(H * L * D, L * D, D), **at):
    a = dict(k=1 * AT, v=2 * AT, cache=3 * AT, slots=4 * AT) | at
    return lib.kv4_append(_ptr(a["k"]), _strides(*ks), _ptr(a["v"]), _strides(*vs), _ptr(a["cache"]), _ptr(a["slots"]),
                          B, H, L, D, PAGES, PAGE, 0, None)


@pytest.mark.parametrize("at", [
    dict(k=3 * AT), dict(v=3 * AT + CACHE - 16), dict(k=3 * AT - ROWS + 16), dict(slots=3 * AT + CACHE - 8),
    dict(slots=3 * AT - 8 * B * L + 8),
    dict(vs=(AT // 2, L * D, D)),                                  # the second sequence's rows begin in the cache
    dict(k=3 * AT + CACHE, ks=(-H * L * D, L * D, D)),             # and these go back into it
    dict(v=3 * AT + CACHE - 16, vs=(0, 0, 0)),                     # one row for every token
], ids=str)
def test_append(lib, at):
    assert append(lib, **at) == pa.ATTN_ERR_SHAPE


HQ = 6
QO = B * HQ * D * 2


def decode(lib, **at):
    need = pa.attn_decode_kv4_workspace_bytes(B, HQ, H, D)
    step = 1 << 26
    assert need < step
    a = {n: (i + 1) * step for i, n in enumerate(("q", "cache", "table", "lens", "o", "slopes", "ws"))}
    a |= {n: (a[f] + d if f else d) for n, (f, d) in at.items()}
    return lib.attn_decode_kv4(_ptr(a["q"]), _ptr(a["cache"]), _ptr(a["table"]), _ptr(a["lens"]), _ptr(a["o"]), B, HQ, H,
                               D, PAGES, PAGE, M, 0.125, _ptr(a["slopes"]), 0.0, 0, _ptr(a["ws"]), need, 0, None)


@pytest.mark.parametrize("at", [
    dict(o=("q", 16)), dict(o=("q", QO - 16)), dict(q=("o", QO - 16)), dict(o=("cache", CACHE - 16)), dict(o=("table", 0)),
    dict(lens=("o", QO - 4)), dict(slopes=("o", 4)), dict(o=("ws", 0)), dict(ws=("o", QO - 16)), dict(ws=("cache", 16)),
    dict(q=("ws", 4096)), dict(table=("ws", 64)), dict(lens=("ws", 4)), dict(slopes=("ws", 8)),
], ids=str)
def test_decode(lib, at):
    assert decode(lib, **at) == pa.ATTN_ERR_SHAPE
