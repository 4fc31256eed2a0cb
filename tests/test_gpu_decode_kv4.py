"""Decode over the paged 4-bit cache against attention in 64 bits over the values it
holds: every kernel, ragged lengths from none on, pages in no order, stale and
missing pages, NaN, far offsets, and the operators run together as they are used."""

import numpy as np
import pytest
import torch

import oracle
import paper_2510_08726_amd as pa
from oracle import serve
from paper_2510_08726_amd.workloads import alibi_slopes, random_tensors
from gpu_common import host64

pytestmark = pytest.mark.gpu

DT = {"f16": torch.float16, "bf16": torch.bfloat16}


def _i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def _cache(lens, Hkv, D, dtype, page, seed, spare=3):
    """A cache of stale bytes with pages in no order; the values of each request as held."""
    rng = np.random.default_rng(seed)
    M = max(-(-int(n) // page) for n in lens) + 1
    total = len(lens) * M + spare
    table = rng.permutation(total)[:len(lens) * M].reshape(len(lens), M)
    cache = torch.randint(0, 256, (total, Hkv, pa.kv4_page_bytes(page, D)), dtype=torch.uint8,
                          generator=torch.Generator().manual_seed(seed)).cuda()
    ks, vs = [], []
    for b, n in enumerate(lens):
        k, v = random_tensors([(1, Hkv, int(n), D)] * 2, dtype, seed + 7 * b + 1)
        if n:
            slots = table[b, np.arange(n) // page] * page + np.arange(n) % page
            pa.kv4_append(k.cuda(), v.cuda(), cache, torch.tensor(slots[None], device="cuda"))
        ks.append(serve.held(host64(k[0]), dtype)[2])
        vs.append(serve.held(host64(v[0]), dtype)[2])
    return cache, table, ks, vs


def _check(o, q, ks, vs, what, *, scale, slopes=None, softcap=None, window=None):
    """Each weight is rounded to the type (half a step of it), and so is the output; scores
    and exponentials in 32 bits are off by under 2e-5 of a weight for scores up to 60
    (60 log2 e 2^-24 and the sums' rounding); fp16 weights under 2^-14 by 2^-25."""
    ref, mean = serve.decode(host64(q), ks, vs, scale=scale, slopes=slopes, softcap=softcap, window=window)
    half = torch.finfo(q.dtype).eps / 2
    most = max([np.abs(v).max() for v in vs if v.size] + [0.0])
    seen = max([min(v.shape[1], window or v.shape[1]) for v in vs] + [0])
    tiny = 2.0 ** -25 * (1 + seen * most) if q.dtype == torch.float16 else 0.0
    tol = half * np.abs(ref) + 1.01 * (half + 2e-5) * mean + tiny + 1e-6
    err = np.abs(host64(o) - ref)
    assert np.isfinite(err).all(), what
    print(f"{what}: worst {np.max(err / tol):.3f} of the tolerance, max abs {err.max():.2e}", flush=True)
    assert (err <= tol).all(), what


def _run(lens, Hq, Hkv, D, dtype, page, seed=0, alibi=False, softcap=None, window=None, scale=None, gain=1.0):
    cache, table, ks, vs = _cache(lens, Hkv, D, dtype, page, seed)
    q, = random_tensors([(len(lens), Hq, 1, D)], dtype, seed + 999)
    q = (q.float() * gain).to(q.dtype)
    sl = alibi_slopes(Hq) if alibi else None
    o = pa.attn_decode_kv4(q.cuda(), cache, _i32(table), _i32(lens), scale=scale, softcap=softcap, window=window,
                           alibi_slopes=None if sl is None else sl.cuda())
    _check(o, q, ks, vs, (lens[:4], Hq, Hkv, D, dtype, page, alibi, softcap, window),
           scale=D ** -0.5 if scale is None else scale, slopes=None if sl is None else host64(sl), softcap=softcap,
           window=window)


@pytest.mark.parametrize("alibi,softcap", [(False, None), (True, None), (False, 2.0), (True, 2.0)])
@pytest.mark.parametrize("Hq,Hkv", [(2, 2), (8, 2), (32, 2), (20, 1), (40, 1)])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
def test_every_kernel(D, dtype, Hq, Hkv, alibi, softcap):
    _run([333, 0, 32, 1, 190], Hq, Hkv, D, dtype, 16, seed=Hq, alibi=alibi, softcap=softcap, gain=4.0 if softcap else 1.0)


@pytest.mark.parametrize("lens", [[0], [1], [0, 0, 5], [16], [31, 32, 33], [15, 17, 63, 64, 65, 127, 128, 129, 257],
                                  [5000], [1, 2, 3] * 40, [0] * 70 + [900] + [0] * 70, [2500, 3, 700, 1]], ids=str)
@pytest.mark.parametrize("page", [16, 32, 128, 1024])
def test_lengths_and_pages(lens, page):
    _run(lens, 8, 2, 128, "bf16", page, seed=page)


@pytest.mark.parametrize("window", [1, 2, 31, 32, 33, 100, 500, 10 ** 9])
@pytest.mark.parametrize("page", [16, 64])
def test_windows(window, page):
    _run([1, 31, 64, 500, 501, 1333], 4, 2, 64, "f16", page, seed=window % 1000, window=window)
    _run([700, 33], 6, 2, 128, "bf16", page, seed=1, window=window, alibi=True)


@pytest.mark.parametrize("scale", [0.0, -0.1, 1.0])
def test_scales(scale):
    _run([77, 300], 8, 4, 64, "bf16", 32, seed=5, scale=scale)


def test_many_shares_of_one_row():
    """One request and one KV head: its row lies in as many shares as there are."""
    _run([40000], 4, 1, 128, "f16", 64, seed=6)
    _run([9000, 1, 9000], 40, 1, 64, "bf16", 256, seed=7)


def test_missing_pages_are_masked():
    lens, page, D = [200, 90], 32, 64
    cache, table, ks, vs = _cache(lens, 2, D, "f16", page, 8)
    q, = random_tensors([(2, 4, 1, D)], "f16", 9)
    t = table.copy()
    t[0, 2], t[0, 4], t[1, 0] = -1, cache.shape[0], 2 ** 31 - 1
    keep = [np.array([t[b, i // page] == table[b, i // page] for i in range(n)]) for b, n in enumerate(lens)]
    o = pa.attn_decode_kv4(q.cuda(), cache, _i32(t), _i32(lens))
    _check(o, q, [k[:, m] for k, m in zip(ks, keep)], [v[:, m] for v, m in zip(vs, keep)], "missing", scale=D ** -0.5)
    o = pa.attn_decode_kv4(q.cuda(), cache, _i32(np.full_like(t, -1)), _i32(lens))     # nothing is left
    assert not o.any()
    # Lengths past the table are clamped, negative ones are empty.
    table = table[:, :2].copy()
    o = pa.attn_decode_kv4(q.cuda(), cache, _i32(table), _i32([10 ** 6, -4]))
    _check(o, q, [ks[0][:, :64], ks[1][:, :0]], [vs[0][:, :64], vs[1][:, :0]], "clamped", scale=D ** -0.5)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_nan_reaches_the_rows_that_see_it(dtype, D):
    lens, page = [70, 70, 70], 16
    cache, table, ks, vs = _cache(lens, 2, D, dtype, page, 10)
    q, = random_tensors([(3, 4, 1, D)], dtype, 11)
    for b, pos in ((0, 20), (1, 69)):       # a V block of head 1, in a full tile and in the last
        x = torch.zeros(1, 2, 1, D, dtype=DT[dtype])
        x[0, 1, 0, 40] = float("inf")
        slot = int(table[b, pos // page]) * page + pos % page
        pa.kv4_append(torch.zeros_like(x).cuda(), x.cuda(), cache, torch.tensor([[slot]], device="cuda"))
    o = pa.attn_decode_kv4(q.cuda(), cache, _i32(table), _i32(lens)).cpu()
    for b in (0, 1):
        assert not o[b, :2].isnan().any() and o[b, 2:, :, 32:64].isnan().all()
        assert not o[b, 2:, :, :32].isnan().any()
    assert not o[2].isnan().any()
    # Out of sight: behind the length, and before the window.
    o = pa.attn_decode_kv4(q.cuda(), cache, _i32(table), _i32([20, 69, 70])).cpu()
    assert not o.isnan().any()
    o = pa.attn_decode_kv4(q.cuda(), cache, _i32(table), _i32([70, 69, 70]), window=49).cpu()
    assert not o.isnan().any()


def test_a_share_of_nan_alone_is_not_left_out():
    """All keys of 300 tokens in the middle are NaN: so whole shares have no maximum."""
    lens, page, D = [3000], 64, 128
    cache, table, _, _ = _cache(lens, 1, D, "bf16", page, 21)
    q, = random_tensors([(1, 2, 1, D)], "bf16", 22, device="cuda")
    x = torch.full((1, 1, 300, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    at = 1000 + np.arange(300)
    pa.kv4_append(x, torch.zeros_like(x), cache, torch.tensor((table[0, at // page] * page + at % page)[None], device="cuda"))
    assert pa.attn_decode_kv4(q, cache, _i32(table), _i32(lens)).isnan().all()
    assert not pa.attn_decode_kv4(q, cache, _i32(table), _i32([1000])).isnan().any()
    assert not pa.attn_decode_kv4(q, cache, _i32(table), _i32(lens), window=1700).isnan().any()


def test_offsets_past_32_bits():
    """Pages behind the first 4 GB of a cache."""
    page, D, Hkv = 256, 128, 8
    block = Hkv * pa.kv4_page_bytes(page, D)
    pages = (1 << 32) // block + 3
    cache = torch.zeros(pages, Hkv, pa.kv4_page_bytes(page, D), dtype=torch.uint8, device="cuda")
    k, v = random_tensors([(1, Hkv, 300, D)] * 2, "bf16", 12)
    q, = random_tensors([(1, 16, 1, D)], "bf16", 13)
    table = np.array([[pages - 1, pages - 3]])
    slots = table[0, np.arange(300) // page] * page + np.arange(300) % page
    pa.kv4_append(k.cuda(), v.cuda(), cache, torch.tensor(slots[None], device="cuda"))
    held = [serve.held(host64(x), "bf16")[2] for x in (k, v)]
    for got, want in zip(pa.kv4_load(cache, _i32(table), _i32([300]), 300, D, torch.bfloat16), held):
        assert np.array_equal(host64(got), want)
    o = pa.attn_decode_kv4(q.cuda(), cache, _i32(table), _i32([300]))
    _check(o, q, [held[0][0]], [held[1][0]], "far", scale=D ** -0.5)


def test_several_query_tokens_by_repeated_rows():
    """Three new tokens of a request are three rows of the call, each with its own length."""
    cache, table, ks, vs = _cache([90], 2, 64, "f16", 16, 14)
    q, = random_tensors([(3, 4, 1, 64)], "f16", 15)
    o = pa.attn_decode_kv4(q.cuda(), cache, _i32(np.repeat(table, 3, 0)), _i32([88, 89, 90]))
    _check(o, q, [ks[0][:, :n] for n in (88, 89, 90)], [vs[0][:, :n] for n in (88, 89, 90)], "tokens", scale=0.125)


def test_calls_repeat_and_do_not_need_a_clean_workspace():
    cache, table, _, _ = _cache([3000, 10, 700], 2, 128, "bf16", 64, 16)
    q, = random_tensors([(3, 16, 1, 128)], "bf16", 17, device="cuda")
    t, n = _i32(table), _i32([3000, 10, 700])
    ws = torch.full((pa.attn_decode_kv4_workspace_bytes(3, 16, 2, 128),), 255, dtype=torch.uint8, device="cuda")
    ref = pa.attn_decode_kv4(q, cache, t, n)
    o = torch.full_like(q, float("nan"))
    assert pa.attn_decode_kv4(q, cache, t, n, o, workspace=ws) is o and torch.equal(o, ref)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    other = pa.attn_decode_kv4(q, cache, t, n, stream=s)
    s.synchronize()
    assert torch.equal(other, ref)


def test_refusals():
    cache, table, _, _ = _cache([20, 30], 2, 64, "f16", 16, 18)
    q, = random_tensors([(2, 4, 1, 64)], "f16", 19, device="cuda")
    t, n = _i32(table), _i32([20, 30])
    sl = alibi_slopes(4).cuda()
    bad = [lambda: pa.attn_decode_kv4(q.float(), cache, t, n), lambda: pa.attn_decode_kv4(q[:, :3].contiguous(), cache, t, n),
           lambda: pa.attn_decode_kv4(q.expand(2, 4, 2, 64).contiguous(), cache, t, n),
           lambda: pa.attn_decode_kv4(q[:1], cache, t, n), lambda: pa.attn_decode_kv4(q, cache, t[:1], n),
           lambda: pa.attn_decode_kv4(q, cache, t, n.long()), lambda: pa.attn_decode_kv4(q, cache, t.cpu(), n),
           lambda: pa.attn_decode_kv4(q, cache[:, :, 16:].contiguous(), t, n), lambda: pa.attn_decode_kv4(q, cache, t, n, q[:1]),
           lambda: pa.attn_decode_kv4(q, cache, t, n, softcap=-1.0), lambda: pa.attn_decode_kv4(q, cache, t, n, window=-1),
           lambda: pa.attn_decode_kv4(q, cache, t, n, scale=float("nan")), lambda: pa.attn_decode_kv4(q, cache, t, n, alibi_slopes=sl[:3]),
           lambda: pa.attn_decode_kv4(q, cache, t, n, alibi_slopes=sl.double()),
           lambda: pa.attn_decode_kv4(q, cache, t, n, workspace=torch.empty(64, dtype=torch.uint8, device="cuda")),
           lambda: pa.attn_decode_kv4(q[:0], cache, t[:0], n[:0])]
    for i, call in enumerate(bad):
        with pytest.raises((ValueError, pa.AttnError)):
            call()
            print("not refused:", i)


@pytest.mark.parametrize("captured", [False, True])
def test_prompts_then_steps(captured):
    """A layer's attention as a serving program runs it: pages and slots of the prompts, rotation,
    append, attention of the prompts over what the cache holds, then decode steps (eagerly, or one
    captured step replayed), each against the definition."""
    B, Hq, Hkv, D, page, L = 3, 8, 2, 64, 16, 50
    M, dtype = 6, "f16"
    counts = np.array([50, 0, 17])
    freqs = serve.frequencies(D, 10000.0)
    f = torch.tensor(freqs, device="cuda")
    table, free = _i32(np.full((B, M), -1)), _i32(np.random.default_rng(0).permutation(B * M))
    cache = torch.full((B * M, Hkv, pa.kv4_page_bytes(page, D)), 255, dtype=torch.uint8, device="cuda")
    lens = _i32([0] * B)

    def step(qkv, counts, lens, free):
        q, k, v = (x.transpose(1, 2) for x in qkv.split([Hq, Hkv, Hkv], 2))
        slots, pos, lens, taken = pa.kv_slots(lens, counts, table, free, page, q.shape[2])
        q, k = pa.rope_fwd(q, k, pos, f)
        pa.kv4_append(k, v, cache, slots)
        return q, k, v, pos, lens, taken

    x, = random_tensors([(B, L, Hq + 2 * Hkv, D)], dtype, 20, device="cuda")
    q, k, v, pos, lens, taken = step(x, _i32(counts), lens, free)
    assert lens.tolist() == counts.tolist() and taken.tolist() == [6] and pos[2, 3] == 3
    held = [[serve.held(host64(t[b, :, :n]), dtype)[2] for b, n in enumerate(counts)] for t in (k, v)]
    for b in (0, 2):
        n = int(counts[b])
        kk, vv = pa.kv4_load(cache, table[b:b + 1], lens[b:b + 1], n, D, DT[dtype])
        assert np.array_equal(host64(kk[0]), held[0][b]) and np.array_equal(host64(vv[0]), held[1][b])
        qb = q[b:b + 1, :, :n].contiguous()
        o = pa.attn_fwd(qb, kk, vv, causal=True)
        ref = oracle.attention(host64(qb), held[0][b][None], held[1][b][None], scale=D ** -0.5, causal=True)
        mean = oracle.attention(host64(qb), held[0][b][None], abs(held[1][b][None]), scale=D ** -0.5, causal=True)
        assert (np.abs(host64(o) - ref) <= 2.0 ** -11 * (np.abs(ref) + 1.01 * mean) + 2e-5 * mean + 2.0 ** -25 * 60).all()

    used = int(taken)
    one = _i32([1] * B)
    x1 = torch.empty(B, 1, Hq + 2 * Hkv, D, dtype=DT[dtype], device="cuda")
    state, stock = lens.clone(), torch.empty(B, dtype=torch.int32, device="cuda")

    def decode():
        q, k, v, pos, new, taken = step(x1, one, state, stock)
        return q, k, v, pos, new, taken, pa.attn_decode_kv4(q, cache, table, new)

    g = None
    if captured:
        stock.copy_(free[used:used + B])
        decode()                                   # what it appends, the first replay appends again
        torch.cuda.synchronize()
        table[:, -(-counts.max() // page):] = -1
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = decode()
    n = counts.copy()
    for s in range(20):
        stock.copy_(free[used:used + B] if used + B <= B * M else torch.cat((free[used:], free[:used + B - B * M])))
        x1.copy_(random_tensors([tuple(x1.shape)], dtype, 30 + s)[0])
        if captured:
            g.replay()
        else:
            out = decode()
        torch.cuda.synchronize()
        q, k, v, pos, new, taken, o = out
        assert pos[:, 0].tolist() == n.tolist() and new.tolist() == (n + 1).tolist()
        want = serve.rope(host64(x1[:, :, :Hq].transpose(1, 2)), n[:, None], freqs)
        assert (np.abs(host64(q) - want) <= 2.0 ** -11 * np.abs(want) + 1e-5).all()
        for b in range(B):
            for h, t in zip(held, (k, v)):
                h[b] = np.concatenate([h[b], serve.held(host64(t[b]), dtype)[2]], 1)
        _check(o, q, held[0], held[1], f"step {s}", scale=D ** -0.5)
        n += 1
        used += int(taken)
        state.copy_(new)
