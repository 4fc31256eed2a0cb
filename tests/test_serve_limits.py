"""Sizes that cannot be launched or represented are refused before anything is enqueued (no GPU).

The C entry points get addresses that are never dereferenced.
"""

import ctypes
import os

import pytest

import paper_2510_08726_amd as pa

AT = [ctypes.c_void_p(i << 42) for i in range(1, 9)]     # far apart: the spans of all operands are disjoint
ZERO = (ctypes.c_longlong * 3)(0, 0, 0)
SHAPE = pa.ATTN_ERR_SHAPE


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(pa.library_path()):
        import __graft_entry__
        __graft_entry__.build()
    return pa.load_library()


@pytest.mark.parametrize("B,Hq,Hkv", [(1 << 18, 64, 64), (1 << 24, 1, 1), (1 << 20, 16, 1), ((1 << 24) // 3 + 1, 3, 3)])
def test_decode_has_a_workgroup_for_each_query_head(lib, B, Hq, Hkv):
    """2^32 threads of 256 a workgroup."""
    assert lib.attn_decode_kv4(*AT[:5], B, Hq, Hkv, 64, 4, 16, 1, 0.1, None, 0.0, 0, AT[5], 1 << 40, 0, None) == SHAPE


@pytest.mark.parametrize("D,L", [(128, ((1 << 24) - 1) * 16 + 1), (64, ((1 << 24) - 1) * 32 + 1), (128, 1 << 30)])
def test_append_and_load_have_a_thread_for_each_vector_of_a_head(lib, D, L):
    """2^32 threads, which hold 8 dims each, of L tokens."""
    assert lib.kv4_append(AT[0], ZERO, AT[1], ZERO, AT[2], AT[3], 1, 1, L, D, 4, 16, 0, None) == SHAPE
    assert lib.kv4_load(*AT[:4], AT[4], AT[5], 1, 1, L, D, 4, 16, 1 << 20, 0, None) == SHAPE


@pytest.mark.parametrize("M,page,L", [(1 << 15, 1 << 15, (1 << 30) + 1), (1, 16, (1 << 31) - 15), (1 << 26, 16, (1 << 31) - 1)])
def test_positions_fit_32_bits(lib, M, page, L):
    assert lib.kv_slots(*AT[:4], 4, 1, M, page, L, *AT[4:8], None) == SHAPE
