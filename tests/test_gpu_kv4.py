"""The paged 4-bit cache on the GPU against the definition: pages and slots, what
is held of every 16-bit value, where it goes, and reading it back."""

import numpy as np
import pytest
import torch

import paper_2510_08726_amd as pa
from oracle import serve
from paper_2510_08726_amd.workloads import random_tensors
from gpu_common import host64

pytestmark = pytest.mark.gpu

DT = {"f16": torch.float16, "bf16": torch.bfloat16}


def _i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def _stale(pages, H, page, D, seed=0):
    g = torch.Generator().manual_seed(seed)
    return torch.randint(0, 256, (pages, H, pa.kv4_page_bytes(page, D)), generator=g, dtype=torch.uint8)


SLOTS = [  # B, L, page, max_pages, longest, share of the free pages
    (1, 1, 16, 1, 0, 1.0), (1, 1, 16, 1, 16, 1.0), (5, 1, 16, 4, 64, 1.0), (3, 40, 16, 5, 60, 1.0),
    (7, 100, 32, 9, 290, 0.5), (300, 1, 64, 3, 190, 0.9), (600, 3, 16, 4, 64, 0.7), (2, 1500, 16, 130, 2000, 1.0),
    (4, 33, 32768, 2, 40000, 1.0), (1030, 1, 16, 2, 32, 0.0),
]


@pytest.mark.parametrize("case", SLOTS, ids=str)
def test_slots(case):
    B, L, page, M, longest, share = case
    rng = np.random.default_rng(B + L)
    lens = rng.integers(0, longest + 1, B)
    lens[rng.random(B) < 0.2] //= page
    lens[rng.random(B) < 0.2] = longest // page * page
    counts = rng.integers(0, L + 1, B)
    table = rng.integers(0, 10 ** 6, (B, M)).astype(np.int32)
    free = rng.permutation(int(B * M * share)).astype(np.int32)
    ref = serve.slots(lens, counts, table, free, page, L)
    t = _i32(table)
    got = pa.kv_slots(_i32(lens), _i32(counts), t, _i32(free), page, L)
    for name, a, b in zip(("slots", "positions", "new_lens", "taken", "table"), (*got, t), ref):
        assert np.array_equal(a.cpu().numpy().reshape(np.shape(b)), b), name
    # Lengths and counts out of range are clamped.
    t = _i32(table)
    got = pa.kv_slots(_i32(lens - 5), _i32(counts + 7 * L), t, _i32(free), page, L)
    ref = serve.slots(lens - 5, np.full(B, L), table, free, page, L) if (counts + 7 * L >= L).all() else None
    for a, b in zip((*got, t), ref):
        assert np.array_equal(a.cpu().numpy().reshape(np.shape(b)), b)


def test_slots_given_outputs_and_refusals():
    lens, counts, table, free = _i32([3, 20]), _i32([2, 1]), _i32([[4, 5], [6, 7]]), _i32([9])
    out = [torch.empty(2, 3, dtype=torch.int64, device="cuda"), torch.empty(2, 3, dtype=torch.int32, device="cuda"),
           torch.empty(2, dtype=torch.int32, device="cuda"), torch.empty(1, dtype=torch.int32, device="cuda")]
    got = pa.kv_slots(lens, counts, table, free, 16, 3, slots=out[0], positions=out[1], new_lens=out[2], taken=out[3])
    assert all(a is b for a, b in zip(got, out)) and out[2].tolist() == [5, 21]
    bad = [lambda: pa.kv_slots(lens, counts, table, free, 16, 3, new_lens=lens),
           lambda: pa.kv_slots(lens, counts, table, free, 16, 3, new_lens=counts),
           lambda: pa.kv_slots(lens, counts, table, free, 17, 3), lambda: pa.kv_slots(lens, counts, table, free, 16, 0),
           lambda: pa.kv_slots(lens.long(), counts, table, free, 16, 3), lambda: pa.kv_slots(lens[:1], counts, table, free, 16, 3),
           lambda: pa.kv_slots(lens, counts, table.t(), free, 16, 3), lambda: pa.kv_slots(lens, counts, table[0], free, 16, 3),
           lambda: pa.kv_slots(lens, counts.cpu(), table, free, 16, 3),
           lambda: pa.kv_slots(lens, counts, table, free, 16, 3, slots=out[1]),
           lambda: pa.kv_slots(lens, counts, table, free, 16, 3, new_lens=out[2], taken=out[2][:1]),
           lambda: pa.kv_slots(table[0], counts, table, free, 16, 3), lambda: pa.kv_slots(lens, counts, table, table[1, 1:], 16, 3)]
    for i, call in enumerate(bad):
        with pytest.raises((ValueError, pa.AttnError)):
            call()
            print("not refused:", i)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
def test_every_value_is_held_as_defined(dtype, D):
    """All 65536 bit patterns, in blocks of like size, in blocks of all sizes, and zeros."""
    bits = np.arange(65536, dtype=np.uint16)
    rng = np.random.default_rng(1)
    rows = np.concatenate([bits, rng.permutation(bits), np.zeros(D, np.uint16)])
    x = torch.from_numpy(rows.view(np.int16)).view(DT[dtype]).reshape(1, 1, -1, D).cuda()
    L, page = x.shape[2], 64
    pages = -(-L // page)
    cache = torch.zeros(pages, 1, pa.kv4_page_bytes(page, D), dtype=torch.uint8, device="cuda")
    slots = torch.arange(L, device="cuda")[None]
    pa.kv4_append(x, x.flip(2), cache, slots)
    table = torch.arange(pages, dtype=torch.int32, device="cuda")[None]
    k, v = pa.kv4_load(cache, table, _i32([L]), L, D, DT[dtype])
    code, scale, value = serve.held(host64(x), dtype)
    for got, want in ((k, value), (v, value[:, :, ::-1])):
        assert np.array_equal(host64(got), want, equal_nan=True)
    ref = np.zeros(cache.shape, np.uint8)
    for t in range(L):
        serve.pack(ref, t, 0, code[0, 0, t], scale[0, 0, t], code[0, 0, L - 1 - t], scale[0, 0, L - 1 - t], page, D)
    got = cache.cpu().numpy()
    assert np.array_equal(got, ref)


CASES = [  # B, H, L, D, dtype, page, pages
    (1, 1, 1, 64, "f16", 16, 1), (2, 3, 5, 128, "bf16", 16, 9), (3, 2, 70, 64, "bf16", 32, 11),
    (2, 5, 33, 128, "f16", 256, 2), (1, 2, 300, 128, "bf16", 32768, 1),
]


@pytest.mark.parametrize("layout", ["plain", "projection"])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_append_and_load(case, layout):
    B, H, L, D, dtype, page, pages = case
    if layout == "plain":
        k, v = random_tensors([(B, H, L, D)] * 2, dtype, 2, device="cuda")
    else:
        x, = random_tensors([(B, L, 3, H, D)], dtype, 2, device="cuda")
        k, v = x[:, :, 1].transpose(1, 2), x[:, :, 2].transpose(1, 2)
    rng = np.random.default_rng(3)
    slots = rng.permutation(pages * page)[:B * L] if pages * page >= B * L else None
    slots = slots.reshape(B, L).astype(np.int64)
    slots[rng.random((B, L)) < 0.2] = -1
    slots.reshape(-1)[-1] = pages * page               # the first that does not exist
    stale = _stale(pages, H, page, D)
    cache = stale.cuda()
    assert pa.kv4_append(k, v, cache, torch.tensor(slots, device="cuda")) is cache
    ref = stale.numpy().copy()
    (ck, sk, _), (cv, sv, _) = serve.held(host64(k), dtype), serve.held(host64(v), dtype)
    for b in range(B):
        for l in range(L):
            if 0 <= slots[b, l] < pages * page:
                for h in range(H):
                    serve.pack(ref, slots[b, l], h, ck[b, h, l], sk[b, h, l], cv[b, h, l], sv[b, h, l], page, D)
    assert np.array_equal(cache.cpu().numpy(), ref)

    # Read back through a table with pages that do not exist, from different starts.
    M = pages + 2
    table = rng.integers(-1, pages + 1, (B, M))
    table[0, :pages] = rng.permutation(pages)
    lens, starts = rng.integers(0, M * page + 1, B), rng.integers(-3, M * page, B)
    lens[0] = M * page + 5
    for st in (None, starts):
        n = min(L + 7, 60)
        got = pa.kv4_load(cache, _i32(table), _i32(lens), n, D, DT[dtype], starts=None if st is None else _i32(st))
        want = np.zeros((2, B, H, n, D))
        for b in range(B):
            for l in range(n):
                t = (0 if st is None else max(st[b], 0)) + l
                if t < min(lens[b], M * page) and 0 <= table[b, t // page] < pages:
                    for h in range(H):
                        want[:, b, h, l] = serve.unpack(ref, table[b, t // page] * page + t % page, h, page, D)
        for a, w in zip(got, want):      # stale scales: beyond the type's range they round to 0 or infinity
            w = torch.from_numpy(w).to(DT[dtype])
            assert torch.equal(a.cpu().nan_to_num(nan=-12345.0), w.nan_to_num(nan=-12345.0))


def test_refusals():
    k, v = random_tensors([(2, 3, 5, 64)] * 2, "f16", 4, device="cuda")
    cache = _stale(4, 3, 16, 64).cuda()
    slots, table, lens = torch.zeros(2, 5, dtype=torch.int64, device="cuda"), _i32([[0, 1], [2, 3]]), _i32([5, 6])
    f16 = torch.float16
    bad = [lambda: pa.kv4_append(k, v[:, :, :4], cache, slots), lambda: pa.kv4_append(k, v.bfloat16(), cache, slots),
           lambda: pa.kv4_append(k.float(), v.float(), cache, slots), lambda: pa.kv4_append(k, v, cache[:, :2].contiguous(), slots),
           lambda: pa.kv4_append(k, v, cache[:, :, :1000].contiguous(), slots), lambda: pa.kv4_append(k, v, cache.int(), slots),
           lambda: pa.kv4_append(k, v, cache, slots.int()), lambda: pa.kv4_append(k, v, cache, slots[:, :4]),
           lambda: pa.kv4_append(k, v, cache.cpu(), slots), lambda: pa.kv4_append(k[..., :32], v[..., :32], cache, slots),
           lambda: pa.kv4_append(k.transpose(2, 3), v.transpose(2, 3), cache, slots),
           lambda: pa.kv4_append(torch.zeros(2, 3, 5, 65, dtype=f16, device="cuda")[..., 1:],
                                 torch.zeros(2, 3, 5, 65, dtype=f16, device="cuda")[..., 1:], cache, slots),
           lambda: pa.kv4_load(cache, table, lens, 5, 64, torch.float32), lambda: pa.kv4_load(cache, table, lens, 0, 64, f16),
           lambda: pa.kv4_load(cache, table, lens[:1], 5, 64, f16), lambda: pa.kv4_load(cache, table.long(), lens, 5, 64, f16),
           lambda: pa.kv4_load(cache, table, lens, 5, 128, f16), lambda: pa.kv4_load(cache, table, lens, 5, 96, f16),
           lambda: pa.kv4_load(cache, table, lens, 5, 64, f16, starts=lens[:1]),
           lambda: pa.kv4_load(cache, table, lens, 5, 64, f16, k, v.bfloat16()),
           lambda: pa.kv4_load(cache, table, lens, 4, 64, f16, k, v)]
    for i, call in enumerate(bad):
        with pytest.raises((ValueError, pa.AttnError)):
            call()
            print("not refused:", i)
