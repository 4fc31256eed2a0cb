"""Operands on another device than the current one: what depends on the device is asked of theirs."""

import pytest
import torch

import paper_2510_08726_amd as pa
from paper_2510_08726_amd.workloads import random_tensors

pytestmark = pytest.mark.gpu


def test_the_decode_sizes_its_workspace_on_the_device_of_q(monkeypatch):
    """The size counts compute units.  One GPU is enough: the size is asked for within the
    context that makes q's device the current one."""
    inside, sizes = [], []

    class Device(torch.cuda.device):
        def __enter__(self):
            inside.append(self.idx)
            return super().__enter__()

        def __exit__(self, *a):
            inside.pop()
            return super().__exit__(*a)

    real = pa.attn_decode_kv4_workspace_bytes

    def size(*a):
        sizes.append(list(inside))
        return real(*a)

    page, D = 16, 64
    q, = random_tensors([(1, 4, 1, D)], "f16", 1, device="cuda")
    cache = torch.zeros(1, 2, pa.kv4_page_bytes(page, D), dtype=torch.uint8, device="cuda")
    table, lens = torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda")
    want = pa.attn_decode_kv4(q, cache, table, lens)
    monkeypatch.setattr(pa, "_BINDING", pa._NotBuilt)
    monkeypatch.setattr(pa, "attn_decode_kv4_workspace_bytes", size)
    monkeypatch.setattr(torch.cuda, "device", Device)
    assert torch.equal(pa.attn_decode_kv4(q, cache, table, lens), want)
    assert sizes == [[q.device.index]]
