"""Operands of the operators around the 4-bit cache that share a buffer: neighbours are
taken, common memory is refused, on both Python paths."""

import pytest
import torch

import paper_2510_08726_amd as pa
from paper_2510_08726_amd.workloads import random_tensors

pytestmark = pytest.mark.gpu


def _shifted(q):
    """A tensor of one sequence that begins eight elements into q."""
    return q.view(-1)[8:8 + q[:1].numel()].view(q[:1].shape)


@pytest.mark.parametrize("path", ["marshalled", "checked"])
def test_neighbours_and_common_memory(monkeypatch, path):
    if path == "checked":
        monkeypatch.setattr(pa, "_BINDING", pa._NotBuilt)
    B, Hq, Hkv, L, D, page, M = 2, 4, 2, 20, 64, 16, 2
    x, = random_tensors([(B, L, 2, Hkv, D)], "f16", 1, device="cuda")
    k, v = x[:, :, 0].transpose(1, 2), x[:, :, 1].transpose(1, 2)
    q, = random_tensors([(B, Hq, 1, D)], "f16", 2, device="cuda")
    cache = torch.zeros(B * M, Hkv, pa.kv4_page_bytes(page, D), dtype=torch.uint8, device="cuda")
    table = torch.arange(B * M, dtype=torch.int32, device="cuda").view(B, M)
    lens = torch.full((B,), L, dtype=torch.int32, device="cuda")
    slots = (table.long()[:, :, None] * page + torch.arange(page, device="cuda")).flatten(1)[:, :L].contiguous()
    pa.kv4_append(k, v, cache, slots)
    a, b = pa.kv4_load(cache, table, lens, L, D, torch.float16)
    o = pa.attn_decode_kv4(q, cache, table, lens)

    both = torch.empty(2, *a.shape, dtype=torch.float16, device="cuda")
    pa.kv4_load(cache, table, lens, L, D, torch.float16, both[0], both[1])
    assert torch.equal(both[0], a) and torch.equal(both[1], b)
    pair = torch.stack((q, torch.zeros_like(q)))
    assert torch.equal(pa.attn_decode_kv4(pair[0], cache, table, lens, pair[1]), o)
    mine = q.clone()
    assert pa.attn_decode_kv4(mine, cache, table, lens, mine) is mine and torch.equal(mine, o)     # in place

    far = torch.zeros(3 * cache.numel(), dtype=torch.uint8, device="cuda")
    shared, rows = far[:cache.numel()].view(cache.shape), far[:2 * a.numel()].view(torch.float16).view(a.shape)
    for call in (lambda: pa.kv4_load(cache, table, lens, L, D, torch.float16, a, a),
                 lambda: pa.kv4_load(shared, table, lens, L, D, torch.float16, rows, b),
                 lambda: pa.kv4_append(rows, v, shared, slots),
                 lambda: pa.attn_decode_kv4(q[:1], cache, table[:1], lens[:1], _shifted(q))):
        with pytest.raises(pa.AttnError) as e:
            call()
        assert e.value.status == pa.ATTN_ERR_SHAPE


@pytest.mark.parametrize("Hq,Hkv,lens", [(8, 2, [5000, 0, 33, 1, 900]), (40, 1, [4000, 4000]), (64, 64, [17] * 40)])
def test_decode_in_place(Hq, Hkv, lens):
    """Rows in one share, in many, and without tokens."""
    D, page, B, M = 128, 64, len(lens), 80
    cache = torch.randint(0, 120, (B * M, Hkv, pa.kv4_page_bytes(page, D)), dtype=torch.uint8,
                          generator=torch.Generator().manual_seed(3)).cuda()
    table = torch.arange(B * M, dtype=torch.int32, device="cuda").view(B, M)
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    q, = random_tensors([(B, Hq, 1, D)], "bf16", 4, device="cuda")
    o = pa.attn_decode_kv4(q, cache, table, n)
    for _ in range(10):
        mine = q.clone()
        pa.attn_decode_kv4(mine, cache, table, n, mine)
        assert torch.equal(mine, o)
