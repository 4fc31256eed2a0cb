"""The operators that write in place, on a stream that is given: what they write is ordered
against the current stream by the caller, here on both sides."""

import numpy as np
import pytest
import torch

import paper_2510_08726_amd as pa
from paper_2510_08726_amd.workloads import random_tensors

pytestmark = pytest.mark.gpu


def _i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def _cases():
    """Name -> (what is written in place, a call on it that returns its outputs)."""
    B, Hkv, L, D, page, M = 40, 4, 300, 128, 16, 40
    rng = np.random.default_rng(0)
    k, v = random_tensors([(B, Hkv, L, D)] * 2, "bf16", 1, device="cuda")
    table, free = _i32(rng.permutation(B * M).reshape(B, M)), _i32(rng.permutation(B * M))
    lens, counts = _i32(rng.integers(0, 300, B)), _i32(rng.integers(0, L + 1, B))
    slots = torch.tensor(rng.permutation(B * M * page)[:B * L].reshape(B, L), device="cuda")
    cache = torch.randint(0, 120, (B * M, Hkv, pa.kv4_page_bytes(page, D)), dtype=torch.uint8,
                          generator=torch.Generator().manual_seed(2)).cuda()
    return {"slots": (table, lambda t, **kw: (*pa.kv_slots(lens, counts, t, free, page, L, **kw), t)),
            "append": (cache, lambda c, **kw: (pa.kv4_append(k, v, c, slots, **kw),))}


@pytest.mark.parametrize("path", ["marshalled", "checked"])
@pytest.mark.parametrize("name", ["slots", "append"])
def test_writes_in_place_on_a_given_stream(monkeypatch, name, path):
    target, call = _cases()[name]
    ref = call(target.clone())
    if path == "checked":
        monkeypatch.setattr(pa, "_BINDING", pa._NotBuilt)
    s = torch.cuda.Stream()
    for r in range(5):
        with torch.cuda.stream(s):           # the copy is made on the call's stream, behind what made its source
            s.wait_stream(torch.cuda.default_stream())
            mine = target.clone()
        out = call(mine, stream=s)
        torch.cuda.current_stream().wait_stream(s)
        assert all(torch.equal(a, b) for a, b in zip(out, ref)), (name, r)
        for t in out:                        # freed on the current stream, behind the comparison
            t.record_stream(torch.cuda.current_stream())
