"""The largest launches that the operators around the 4-bit cache take."""

import pytest
import torch

import paper_2510_08726_amd as pa
from paper_2510_08726_amd.workloads import random_tensors

pytestmark = pytest.mark.gpu


def test_append_of_the_most_tokens():
    """2^24 - 1 workgroups of 16 tokens; K and V are one row for every token, and one slot is real."""
    D, L, page = 128, ((1 << 24) - 1) * 16, 16
    k, v = random_tensors([(1, 1, 1, D)] * 2, "bf16", 1, device="cuda")
    slots = torch.full((1, L), -1, dtype=torch.int64, device="cuda")
    slots[0, L - 1] = 21
    cache, want = (torch.zeros(2, 1, pa.kv4_page_bytes(page, D), dtype=torch.uint8, device="cuda") for _ in range(2))
    pa.kv4_append(k.expand(1, 1, L, D), v.expand(1, 1, L, D), cache, slots)
    pa.kv4_append(k, v, want, slots[:, L - 1:].contiguous())
    assert want.any() and torch.equal(cache, want)


def test_decode_of_the_most_heads():
    """2^24 - 64 query heads; the last sequence alone has tokens."""
    B, H, D, page = (1 << 18) - 1, 64, 64, 16
    k, v, q1 = random_tensors([(1, H, 3, D), (1, H, 3, D), (1, H, 1, D)], "f16", 2, device="cuda")
    cache = torch.zeros(1, H, pa.kv4_page_bytes(page, D), dtype=torch.uint8, device="cuda")
    pa.kv4_append(k, v, cache, torch.arange(3, device="cuda")[None])
    q = torch.zeros(B, H, 1, D, dtype=torch.float16, device="cuda")
    q[-1] = q1[0]
    table, lens = torch.zeros(B, 1, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
    lens[-1] = 3
    o = pa.attn_decode_kv4(q, cache, table, lens)
    assert torch.equal(o[-1:], pa.attn_decode_kv4(q1, cache, table[:1], lens[-1:].contiguous()))
    assert o[-1].any() and not o[:-1].any()
