"""What the operators of a training step refuse, on the host (no GPU).

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
NULL, SHAPE, UNSUPPORTED, WORKSPACE = pa.ATTN_ERR_NULL, pa.ATTN_ERR_SHAPE, pa.ATTN_ERR_UNSUPPORTED, pa.ATTN_ERR_WORKSPACE
INF, NAN = float("inf"), float("nan")


def at(n, off=0):
    """A pointer 2^40 bytes from the others."""
    return ctypes.c_void_p((n << 40) + off)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(pa.library_path()):
        import __graft_entry__
        __graft_entry__.build()
    return pa.load_library()


def test_every_declared_symbol_is_exported(lib):
    for h, n in (("attn_bwd.h", 3), ("rmsnorm.h", 5)):
        src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", h)).read(), flags=re.S)
        names = re.findall(r"\b((?:attn|rmsnorm|quant8)_[a-z0-9_]+)\s*\(", src)
        assert len(names) == n
        for name in names:
            assert hasattr(lib, name) and name in pa.__all__, name


SIZES = dict(B=2, Hq=4, Hkv=2, Lq=32, Lk=48, D=64)
MOD = dict(causal=1, scale=0.125, slopes=None, softcap=0.0, window=0)


def fwd(lib, q=at(1), k=at(2), v=at(3), o=at(4), lse=at(5), dtype=0, **kw):
    s, m = {**SIZES, **{x: kw[x] for x in SIZES if x in kw}}, {**MOD, **{x: kw[x] for x in MOD if x in kw}}
    return lib.attn_fwd_lse(q, k, v, o, lse, *s.values(), m["causal"], m["scale"], m["slopes"], m["softcap"], m["window"],
                            dtype, None)


def strides(*s):
    return (ctypes.c_longlong * 3)(*s)


def bwd(lib, do=at(1), ds=strides(8192, 2048, 64), q=at(2), k=at(3), v=at(4), o=at(5), lse=at(6), dq=at(7), dk=at(8), dv=at(9),
        ws=at(10), size=None, dtype=0, **kw):
    s, m = {**SIZES, **{x: kw[x] for x in SIZES if x in kw}}, {**MOD, **{x: kw[x] for x in MOD if x in kw}}
    if size is None:
        size = lib.attn_bwd_workspace_bytes(*s.values(), m["causal"], m["window"])
    return lib.attn_bwd(do, ds, q, k, v, o, lse, dq, dk, dv, *s.values(), m["causal"], m["scale"], m["slopes"], m["softcap"],
                        m["window"], ws, size, dtype, None)


BOTH = [
    (dict(B=0), SHAPE), (dict(Hq=0), SHAPE), (dict(Hkv=0), SHAPE), (dict(Lq=0), SHAPE), (dict(Lk=0), SHAPE), (dict(Hq=3), SHAPE),
    (dict(D=96), UNSUPPORTED), (dict(D=0), UNSUPPORTED), (dict(dtype=2), UNSUPPORTED), (dict(dtype=-1), UNSUPPORTED),
    (dict(scale=NAN), SHAPE), (dict(scale=INF), SHAPE), (dict(softcap=-1.0), SHAPE), (dict(softcap=NAN), SHAPE),
    (dict(window=-1), SHAPE), (dict(window=4, causal=0), UNSUPPORTED), (dict(softcap=5.0, causal=0), UNSUPPORTED),
    (dict(softcap=5.0, slopes=at(20)), UNSUPPORTED), (dict(softcap=1025.0), UNSUPPORTED),
    (dict(Lq=1 << 24), SHAPE), (dict(Lk=(1 << 24) - 16), SHAPE), (dict(B=1 << 20, Hq=1 << 12, Hkv=1 << 12), SHAPE),
    (dict(Lq=1 << 23, Hq=1 << 6, Hkv=1), SHAPE),
]


@pytest.mark.parametrize("kw,code", BOTH + [
    (dict(q=None), NULL), (dict(k=None), NULL), (dict(v=None), NULL), (dict(o=None), NULL), (dict(lse=None), NULL),
    (dict(o=at(1)), SHAPE), (dict(o=at(2)), SHAPE), (dict(o=at(3, 64)), SHAPE), (dict(lse=at(1)), SHAPE), (dict(lse=at(4)), SHAPE),
    (dict(slopes=at(4)), SHAPE), (dict(slopes=at(5)), SHAPE),
], ids=str)
def test_attn_fwd_lse(lib, kw, code):
    assert fwd(lib, **kw) == code


@pytest.mark.parametrize("kw,code", BOTH + [
    *[({name: None}, NULL) for name in ("do", "ds", "q", "k", "v", "o", "lse", "dq", "dk", "dv", "ws")],
    *[({name: at(n, 8)}, SHAPE) for n, name in enumerate(("do", "q", "k", "v", "o"), 1) for n in (n if name == "do" else n,)],
    (dict(dq=at(7, 8)), SHAPE), (dict(dk=at(8, 2)), SHAPE), (dict(dv=at(9, 4)), SHAPE),
    (dict(ds=strides(8192, 2048, 65)), SHAPE), (dict(ds=strides(8192, 2048, -64)), SHAPE), (dict(ds=strides(8196, 2048, 64)), SHAPE),
    (dict(ds=strides(8192, 2048, 1 << 26)), SHAPE), (dict(ds=strides(1 << 40, 2048, 64)), SHAPE),
    (dict(dq=at(1)), SHAPE), (dict(dq=at(2)), SHAPE), (dict(dk=at(3)), SHAPE), (dict(dv=at(4)), SHAPE), (dict(dq=at(5)), SHAPE),
    (dict(dk=at(6)), SHAPE), (dict(dk=at(7)), SHAPE), (dict(dv=at(8, 1024)), SHAPE), (dict(ws=at(9)), SHAPE), (dict(ws=at(2)), SHAPE),
    (dict(slopes=at(10)), SHAPE), (dict(slopes=at(7, 16)), SHAPE),
    (dict(ds=strides(8192, 2048, 1024), dq=at(1, 31 * 2048 + 64)), SHAPE),       # within what the strides reach
    (dict(size=16), WORKSPACE), (dict(size=0), WORKSPACE), (dict(ws=at(10, 8)), WORKSPACE),
], ids=str)
def test_attn_bwd(lib, kw, code):
    assert bwd(lib, **kw) == code


def test_workspace_sizes(lib):
    size = lambda **kw: lib.attn_bwd_workspace_bytes(*{**SIZES, **kw}.values(), 1, 0)     # noqa: E731
    assert size() > 0
    for kw in (dict(B=0), dict(D=96), dict(Hq=3), dict(Lk=0), dict(Lq=1 << 24)):
        assert size(**kw) == 0, kw
    assert lib.attn_bwd_workspace_bytes(*SIZES.values(), 1, -1) == 0
    assert pa.attn_bwd_workspace_bytes(1 << 32, 4, 2, 32, 48, 64) == 0
    assert pa.attn_bwd_workspace_bytes(2, 4, 2, 32, 48, 64, True, 1 << 40) == size()
    # Partials: at most two for each workgroup that a device holds (256 compute units here), and one for each
    # block that is divided.
    most = 2 * 3 * 512 * 128 * 128 * 4 * 2
    for B, Hq, Hkv, L in ((1, 1, 1, 1 << 15), (2, 32, 8, 2048), (1, 40, 2, 2048), (1, 64, 1, 300), (1, 32, 8, 128)):
        for causal in (0, 1):
            assert lib.attn_bwd_workspace_bytes(B, Hq, Hkv, L, 8192, 128, causal, 0) <= most
    assert lib.rmsnorm_add_bwd_workspace_bytes(0, 64) == 0 and lib.rmsnorm_add_bwd_workspace_bytes(5, 1 << 20) == 0
    assert lib.rmsnorm_add_bwd_workspace_bytes(5, 64) >= 5 // 4 * 64 * 4
    assert pa.rmsnorm_add_bwd_workspace_bytes(1 << 40, 64) == 0


def norm(lib, x=at(1), res=at(2), w=at(3), y=at(4), h=at(5), rstd=at(6), N=8, M=64, eps=1e-6, off=0.0, dtype=0, wide=0):
    return lib.rmsnorm_add(x, res, w, y, h, rstd, N, M, eps, off, dtype, wide, None)


def quant(lib, x=at(1), res=at(2), w=at(3), y=at(4), sc=at(7), h=at(5), rstd=at(6), N=8, M=64, group=0, code=0, eps=1e-6,
          off=0.0, dtype=0, wide=0):
    return lib.rmsnorm_add_quant(x, res, w, y, sc, h, rstd, N, M, group, code, eps, off, dtype, wide, None)


NORMS = [
    (dict(x=None), NULL), (dict(y=None), NULL), (dict(h=None), NULL),
    (dict(N=0), SHAPE), (dict(M=0), SHAPE), (dict(M=32769), SHAPE), (dict(N=1 << 30, M=1 << 10), SHAPE),
    (dict(eps=-1.0), SHAPE), (dict(eps=NAN), SHAPE), (dict(off=INF), SHAPE),
    (dict(dtype=3), UNSUPPORTED), (dict(dtype=-1), UNSUPPORTED), (dict(dtype=0, wide=1), UNSUPPORTED),
    (dict(dtype=2, wide=0), UNSUPPORTED), (dict(res=None, wide=2), UNSUPPORTED),
    (dict(h=at(1)), SHAPE), (dict(h=at(2, 16)), SHAPE), (dict(h=at(3)), SHAPE), (dict(rstd=at(1)), SHAPE), (dict(rstd=at(5)), SHAPE),
    (dict(y=at(2)), SHAPE), (dict(y=at(3)), SHAPE), (dict(y=at(5)), SHAPE), (dict(y=at(6)), SHAPE), (dict(y=at(1, 2)), SHAPE),
    (dict(wide=2, h=at(2, 8)), SHAPE),
]


@pytest.mark.parametrize("kw,code", NORMS, ids=str)
def test_rmsnorm_add(lib, kw, code):
    assert norm(lib, **kw) == code
    assert quant(lib, **kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(sc=None), NULL), (dict(code=2), UNSUPPORTED), (dict(code=-1), UNSUPPORTED), (dict(group=16), SHAPE),
    (dict(group=-1), SHAPE), (dict(group=512), SHAPE), (dict(y=at(1)), SHAPE), (dict(sc=at(4)), SHAPE), (dict(sc=at(2)), SHAPE),
    (dict(sc=at(6)), SHAPE), (dict(group=32, sc=at(6, -40)), SHAPE),
], ids=str)
def test_rmsnorm_add_quant(lib, kw, code):
    assert quant(lib, **kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(q=None), NULL), (dict(s=None), NULL), (dict(y=None), NULL), (dict(N=0), SHAPE), (dict(M=40000), SHAPE),
    (dict(group=8), SHAPE), (dict(code=5), UNSUPPORTED), (dict(dtype=7), UNSUPPORTED), (dict(y=at(1)), SHAPE), (dict(y=at(2)), SHAPE),
], ids=str)
def test_quant8_load(lib, kw, code):
    a = {**dict(q=at(1), s=at(2), y=at(3), N=8, M=64, group=0, code=0, dtype=0), **kw}
    assert lib.quant8_load(*a.values(), None) == code


@pytest.mark.parametrize("kw,code", [
    (dict(dy=None), NULL), (dict(h=None), NULL), (dict(rstd=None), NULL), (dict(dx=None), NULL),
    (dict(N=0), SHAPE), (dict(M=0), SHAPE), (dict(M=32769), SHAPE), (dict(off=NAN), SHAPE),
    (dict(dtype=3), UNSUPPORTED), (dict(wide=1), UNSUPPORTED),
    (dict(dres=at(9)), SHAPE),                                            # of dX's type: dX is that
    (dict(ws=None), WORKSPACE), (dict(size=16), WORKSPACE), (dict(ws=at(8, 8)), WORKSPACE),
    (dict(dx=at(2)), SHAPE), (dict(dx=at(3)), SHAPE), (dict(dx=at(4)), SHAPE), (dict(dx=at(5, 16)), SHAPE), (dict(dx=at(1, 16)), SHAPE),
    (dict(dw=at(1)), SHAPE), (dict(dw=at(4)), SHAPE), (dict(dw=at(6)), SHAPE), (dict(ws=at(2)), SHAPE), (dict(ws=at(6)), SHAPE),
    (dict(wide=2, dres=at(6)), SHAPE), (dict(wide=2, dres=at(1)), SHAPE), (dict(wide=2, dx=at(5)), SHAPE),
    (dict(wide=2, dres=at(5, 16)), SHAPE),
], ids=str)
def test_rmsnorm_add_bwd(lib, kw, code):
    a = {**dict(dy=at(1), h=at(2), rstd=at(3), w=at(4), dh=at(5), dx=at(6), dres=None, dw=at(7), N=8, M=64, off=0.0, ws=at(8),
                size=1 << 20, dtype=0, wide=0), **kw}
    assert lib.rmsnorm_add_bwd(*a.values(), None) == code


def test_tensors_on_the_host_are_refused():
    q = torch.zeros(1, 2, 8, 64, dtype=torch.float16)
    lse = torch.zeros(1, 2, 8)
    x = torch.zeros(4, 64)
    for call in (lambda: pa.attn_fwd_lse(q, q, q), lambda: pa.attn_bwd(q, q, q, q, q, lse), lambda: pa.rmsnorm_add(x),
                 lambda: pa.rmsnorm_add_quant(x), lambda: pa.quant8_load(x.to(torch.int8), lse),
                 lambda: pa.rmsnorm_add_bwd(x, x, x[:, 0])):
        with pytest.raises(ValueError):
            call()
