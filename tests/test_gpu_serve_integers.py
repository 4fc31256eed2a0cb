"""Integers that 32 bits do not hold: a window that wide sees everything, sizes are refused."""

import pytest
import torch

import paper_2510_08726_amd as pa
from paper_2510_08726_amd.workloads import random_tensors

pytestmark = pytest.mark.gpu

BIG = 1 << 32


def test_window_and_sizes():
    B, Hq, Hkv, L, D, page = 2, 4, 2, 40, 64, 16
    k, v = random_tensors([(B, Hkv, L, D)] * 2, "f16", 1, device="cuda")
    q, = random_tensors([(B, Hq, 1, D)], "f16", 2, device="cuda")
    cache = torch.zeros(6, Hkv, pa.kv4_page_bytes(page, D), dtype=torch.uint8, device="cuda")
    table = torch.arange(6, dtype=torch.int32, device="cuda").view(B, 3)
    lens = torch.full((B,), L, dtype=torch.int32, device="cuda")
    pa.kv4_append(k, v, cache, torch.arange(B * 48, device="cuda").view(B, 48)[:, :L].contiguous())
    all_of_it = pa.attn_decode_kv4(q, cache, table, lens)
    for window in (BIG + 5, BIG, 1 << 31, (1 << 31) - 1):
        assert torch.equal(pa.attn_decode_kv4(q, cache, table, lens, window=window), all_of_it), window
    counts, free = torch.zeros_like(lens), torch.arange(3, dtype=torch.int32, device="cuda")
    out = dict(slots=torch.zeros(B, 1, dtype=torch.int64, device="cuda"),
               positions=torch.zeros(B, 1, dtype=torch.int32, device="cuda"))
    for call in (lambda: pa.attn_decode_kv4(q, cache, table, lens, window=5 - BIG),
                 lambda: pa.kv_slots(lens, counts, table, free, BIG + page, 1),
                 lambda: pa.kv_slots(lens, counts, table, free, page, BIG + 1, **out),
                 lambda: pa.kv4_load(cache, table, lens, BIG + L, D, torch.float16, k, v),
                 lambda: pa.kv4_load(cache, table, lens, L, BIG + D, torch.float16)):
        with pytest.raises((ValueError, pa.AttnError)):
            call()
