"""What the operators around the 4-bit cache refuse, on the host (no GPU).

The C entry points get pointers that are never dereferenced: every call here
fails validation, which runs before anything is enqueued.
"""

import ctypes
import os
import re

import pytest
import torch

import paper_2510_08726_amd as pa

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE, OTHER, ODD = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x2000), ctypes.c_void_p(0x1008)
OK, NULL, SHAPE, UNSUPPORTED, WORKSPACE = 0, pa.ATTN_ERR_NULL, pa.ATTN_ERR_SHAPE, pa.ATTN_ERR_UNSUPPORTED, pa.ATTN_ERR_WORKSPACE


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(pa.library_path()):
        import __graft_entry__
        __graft_entry__.build()
    return pa.load_library()


def test_every_declared_symbol_is_exported(lib):
    for h in ("rope.h", "kv4.h"):
        src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", h)).read(), flags=re.S)
        names = re.findall(r"\b((?:rope|kv4|kv|attn)_[a-z0-9_]+)\s*\(", src)
        assert len(names) >= 3
        for n in names:
            assert hasattr(lib, n) and n in pa.__all__, n


def strides(*s):
    return (ctypes.c_longlong * 3)(*s)


def rope(lib, q=FAKE, qs=strides(0, 0, 0), qo=FAKE, Hq=2, k=FAKE, ks=strides(0, 0, 0), ko=FAKE, Hkv=2, B=1, L=1, D=64,
         pos=FAKE, bits=32, pstride=0, f=FAKE, R=64, inter=0, mag=1.0, dtype=0):
    a = (q, qs, qo, Hq, k, ks, ko, Hkv, B, L, D, pos, bits, pstride, f, R, inter, mag, dtype, None)
    rc = lib.rope_fwd(*a)
    assert lib.rope_bwd(*a) == rc
    return rc


@pytest.mark.parametrize("kw,code", [
    (dict(q=None), NULL), (dict(qs=None), NULL), (dict(qo=None), NULL), (dict(pos=None), NULL), (dict(f=None), NULL),
    (dict(ks=None), NULL), (dict(ko=None), NULL),
    (dict(k=None), SHAPE), (dict(Hkv=0), SHAPE), (dict(Hq=0), SHAPE), (dict(B=0), SHAPE), (dict(L=0), SHAPE),
    (dict(D=1, R=2), SHAPE), (dict(R=0), SHAPE), (dict(R=63), SHAPE), (dict(R=66), SHAPE),
    (dict(mag=float("nan")), SHAPE), (dict(mag=float("inf")), SHAPE), (dict(bits=16), SHAPE), (dict(pstride=-1), SHAPE),
    (dict(B=1 << 20, L=1 << 20), SHAPE), (dict(B=1 << 15, L=1 << 15, D=1 << 10), SHAPE), (dict(Hq=70000), SHAPE),
    (dict(dtype=3), UNSUPPORTED), (dict(dtype=-1), UNSUPPORTED),
], ids=str)
def test_rope(lib, kw, code):
    assert rope(lib, **kw) == code


def test_rope_frequencies(lib):
    buf = (ctypes.c_double * 8)()
    f = lambda R=16, base=1e4, s=0, factor=2.0, n=100.0, slow=1.0, fast=4.0, out=buf: lib.rope_frequencies(  # noqa: E731
        R, base, s, factor, n, slow, fast, out)
    assert f() == OK and f(out=None) == NULL and f(s=4) == UNSUPPORTED and f(s=-1) == UNSUPPORTED
    for kw in (dict(R=0), dict(R=15), dict(base=0.0), dict(base=float("inf")), dict(s=1, factor=0.0), dict(R=2, s=2),
               dict(s=3, n=0.0), dict(s=3, slow=4.0), dict(s=3, slow=-1.0), dict(s=3, fast=float("nan"))):
        assert f(**kw) == SHAPE, kw
    assert f(factor=0.0) == OK                     # no scaling: not looked at
    with pytest.raises(ValueError):
        pa.rope_frequencies(16, scaling="other")
    with pytest.raises(pa.AttnError):
        pa.rope_frequencies(15)


def slots(lib, lens=FAKE, counts=FAKE, table=FAKE, free=FAKE, F=4, B=2, M=3, page=16, L=5, s=FAKE, p=FAKE, n=OTHER,
          t=FAKE):
    return lib.kv_slots(lens, counts, table, free, F, B, M, page, L, s, p, n, t, None)


@pytest.mark.parametrize("kw,code", [
    (dict(lens=None), NULL), (dict(counts=None), NULL), (dict(table=None), NULL), (dict(free=None), NULL),
    (dict(s=None), NULL), (dict(p=None), NULL), (dict(n=None), NULL), (dict(t=None), NULL),
    (dict(n=FAKE), SHAPE),                         # new_lens is lens
    (dict(B=0), SHAPE), (dict(M=0), SHAPE), (dict(L=0), SHAPE), (dict(F=-1), SHAPE),
    (dict(page=8), SHAPE), (dict(page=24), SHAPE), (dict(page=0), SHAPE), (dict(page=-16), SHAPE), (dict(page=65536), SHAPE),
    (dict(B=1 << 16, L=1 << 16), SHAPE), (dict(B=1 << 16, M=1 << 16), SHAPE), (dict(M=1 << 27), SHAPE),
], ids=str)
def test_slots(lib, kw, code):
    assert slots(lib, **kw) == code


def append(lib, k=FAKE, ks=strides(0, 0, 0), v=FAKE, vs=strides(0, 0, 0), c=FAKE, s=FAKE, B=1, H=2, L=3, D=64, P=4,
           page=16, dtype=0):
    return lib.kv4_append(k, ks, v, vs, c, s, B, H, L, D, P, page, dtype, None)


def load(lib, c=FAKE, t=FAKE, st=None, n=FAKE, k=FAKE, v=FAKE, B=1, H=2, L=3, D=64, P=4, page=16, M=3, dtype=0):
    return lib.kv4_load(c, t, st, n, k, v, B, H, L, D, P, page, M, dtype, None)


@pytest.mark.parametrize("kw,code", [
    (dict(k=None), NULL), (dict(v=None), NULL), (dict(c=None), NULL),
    (dict(B=0), SHAPE), (dict(H=0), SHAPE), (dict(L=0), SHAPE), (dict(P=0), SHAPE), (dict(page=48), SHAPE),
    (dict(k=ODD), SHAPE), (dict(v=ODD), SHAPE), (dict(c=ODD), SHAPE), (dict(B=1 << 16, H=1 << 10, L=1 << 12), SHAPE), (dict(H=1 << 16), SHAPE),
    (dict(D=96), UNSUPPORTED), (dict(D=32), UNSUPPORTED), (dict(dtype=2), UNSUPPORTED),
], ids=str)
def test_append_and_load(lib, kw, code):
    assert append(lib, **kw) == code and load(lib, **kw) == code


def test_append_strides_and_load_tables(lib):
    assert append(lib, s=None) == NULL and append(lib, ks=None) == NULL and append(lib, vs=None) == NULL
    assert append(lib, ks=strides(64, 4, 64)) == SHAPE and append(lib, vs=strides(0, 0, 66)) == SHAPE
    assert load(lib, t=None) == NULL and load(lib, n=None) == NULL
    assert load(lib, M=0) == SHAPE and load(lib, M=1 << 27) == SHAPE


def decode(lib, q=FAKE, c=FAKE, t=FAKE, n=FAKE, o=FAKE, B=2, Hq=8, Hkv=2, D=128, P=4, page=16, M=3, scale=0.1,
           slopes=None, cap=0.0, window=0, ws=FAKE, bytes=1 << 30, dtype=0):
    return lib.attn_decode_kv4(q, c, t, n, o, B, Hq, Hkv, D, P, page, M, scale, slopes, cap, window, ws, bytes, dtype,
                               None)


@pytest.mark.parametrize("kw,code", [
    (dict(q=None), NULL), (dict(c=None), NULL), (dict(t=None), NULL), (dict(n=None), NULL), (dict(o=None), NULL),
    (dict(ws=None), NULL),
    (dict(B=0), SHAPE), (dict(Hq=0), SHAPE), (dict(Hkv=0), SHAPE), (dict(Hq=6, Hkv=4), SHAPE), (dict(P=0), SHAPE),
    (dict(M=0), SHAPE), (dict(page=17), SHAPE), (dict(window=-1), SHAPE), (dict(scale=float("nan")), SHAPE),
    (dict(cap=-1.0), SHAPE), (dict(cap=float("inf")), SHAPE), (dict(M=1 << 27), SHAPE),
    (dict(B=1 << 10, Hkv=1 << 7, Hq=1 << 7, M=1 << 20), SHAPE),
    (dict(q=ODD), SHAPE), (dict(o=ODD), SHAPE), (dict(c=ODD), SHAPE),
    (dict(D=96), UNSUPPORTED), (dict(dtype=5), UNSUPPORTED),
    (dict(bytes=100), WORKSPACE), (dict(ws=ODD), WORKSPACE),
], ids=str)
def test_decode(lib, kw, code):
    assert decode(lib, **kw) == code


def test_sizes(lib):
    assert pa.kv4_page_bytes(64, 128) == 64 * 136 and pa.kv4_page_bytes(16, 64) == 16 * 68
    for bad in ((8, 64), (48, 64), (65536, 64), (16, 96), (0, 64)):
        assert pa.kv4_page_bytes(*bad) == 0
    a, b = (pa.attn_decode_kv4_workspace_bytes(n, 8, 2, 128) for n in (1, 64))
    assert 0 < a <= b <= a + 64 * 2 * 8              # 8 bytes a row beside what the device needs
    for bad in ((0, 8, 2, 128), (1, 7, 2, 128), (1, 8, 2, 96), (1, 8, 0, 64)):
        assert pa.attn_decode_kv4_workspace_bytes(*bad) == 0
    need = pa.attn_decode_kv4_workspace_bytes(2, 8, 2, 128)
    assert decode(lib, bytes=need - 1) == WORKSPACE


def test_cpu_tensors_are_refused():
    x = torch.zeros(1, 2, 3, 64, dtype=torch.float16)
    i, l = torch.zeros(1, dtype=torch.int32), torch.zeros(1, 3, dtype=torch.int64)
    cache, table = torch.zeros(2, 2, 1088, dtype=torch.uint8), torch.zeros(1, 2, dtype=torch.int32)
    for f in (lambda: pa.rope_fwd(x, x, l, torch.ones(32, dtype=torch.float64)),
              lambda: pa.rope_bwd(x, None, l, torch.ones(32, dtype=torch.float64)),
              lambda: pa.kv_slots(i, i, table, i, 16, 3), lambda: pa.kv4_append(x, x, cache, l),
              lambda: pa.kv4_load(cache, table, i, 3, 64, torch.float16),
              lambda: pa.attn_decode_kv4(x[:, :, :1].contiguous(), cache, table, i)):
        with pytest.raises(ValueError):
            f()
