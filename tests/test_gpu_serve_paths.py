"""The serving operators on every Python path: marshalled in C++, through the Python checks,
on a stream that is given, captured in a graph; and two calls at once."""

import numpy as np
import pytest
import torch

import paper_2510_08726_amd as pa
from paper_2510_08726_amd.workloads import alibi_slopes, random_tensors

pytestmark = pytest.mark.gpu


def _i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def _calls():
    """Name -> a call that returns its outputs (and leaves its inputs as they were)."""
    B, Hq, Hkv, L, D, page, M = 3, 6, 2, 5, 64, 16, 7
    x, = random_tensors([(B, L, Hq + 2 * Hkv, D)], "f16", 1, device="cuda")
    q, k, v = (t.transpose(1, 2) for t in x.split([Hq, Hkv, Hkv], 2))
    f = pa.rope_frequencies(48, scaling="base", factor=2.0, device="cuda")
    pos = torch.arange(B * L, device="cuda").view(B, L)
    lens, counts = _i32([70, 0, 33]), _i32([5, 2, 0])
    table, free = _i32(np.random.default_rng(0).permutation(B * M).reshape(B, M)), _i32([3, 1, 2])
    cache = torch.randint(0, 120, (B * M, Hkv, pa.kv4_page_bytes(page, D)), dtype=torch.uint8,
                          generator=torch.Generator().manual_seed(2)).cuda()
    slots = torch.tensor(np.random.default_rng(3).permutation(B * M * page)[:B * L].reshape(B, L), device="cuda")
    one, = random_tensors([(B, Hq, 1, D)], "f16", 4, device="cuda")
    sl, starts = alibi_slopes(Hq).cuda(), _i32([50, 0, 3])

    def place(**kw):
        t = table.clone()
        return (*pa.kv_slots(lens, counts, t, free, page, L, **kw), t)

    return {
        "rope": lambda **kw: pa.rope_fwd(q, k, pos, f, interleaved=True, magnitude=1.25, **kw),
        "rope one": lambda **kw: pa.rope_bwd(q, None, pos[1], f, **kw)[:1],
        "slots": place,
        "append": lambda **kw: (pa.kv4_append(k, v, cache.clone(), slots, **kw),),
        "load": lambda **kw: pa.kv4_load(cache, table, lens, 40, D, torch.float16, starts=starts, **kw),
        "load all": lambda **kw: pa.kv4_load(cache, table, lens, 70, D, torch.bfloat16, **kw),
        "decode": lambda **kw: (pa.attn_decode_kv4(one, cache, table, lens, **kw),),
        "decode modified": lambda **kw: (pa.attn_decode_kv4(one, cache, table, lens, scale=0.2, alibi_slopes=sl,
                                                            softcap=3.0, window=40, **kw),),
    }


def _same(a, b):
    return len(a) == len(b) and all(x.dtype == y.dtype and torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("name", list(range(8)))
def test_every_path(monkeypatch, name):
    name, call = list(_calls().items())[name]
    ref = call()
    assert not any(t.is_floating_point() and t.isnan().any() for t in ref), name
    with monkeypatch.context() as m:
        m.setattr(pa, "_BINDING", pa._NotBuilt)
        assert _same(call(), ref), name
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    other = call(stream=s)
    s.synchronize()
    assert _same(other, ref), name
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = call()
    for r in range(4):
        for t in out:
            t.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert _same(out, ref), (name, r)
        call()


def test_two_decodes_at_once():
    """Calls that overlap on two streams have workspaces of their own."""
    torch.manual_seed(0)
    page, D, H = 64, 128, 8
    n = [9000, 4000]
    caches = [torch.randint(0, 120, (150, H, pa.kv4_page_bytes(page, D)), dtype=torch.uint8, device="cuda") for _ in n]
    qs = [torch.randn(1, 32, 1, D, device="cuda", dtype=torch.bfloat16) for _ in n]
    table = torch.randperm(150, device="cuda").to(torch.int32)[None].contiguous()
    lens = [_i32([x]) for x in n]
    ref = [pa.attn_decode_kv4(q, c, table, x) for q, c, x in zip(qs, caches, lens)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in n]
    got = [[], []]
    for _ in range(20):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(pa.attn_decode_kv4(qs[i], caches[i], table, lens[i]))
    torch.cuda.synchronize()
    assert all(torch.equal(o, r) for outs, r in zip(got, ref) for o in outs)
