"""The serving operators around attention over a 4-bit cache: what is timed, and their plain forms.

Rotary positions (``rope_fwd``, ``rope_bwd``), the pages and slots of new tokens (``kv_slots``),
the 4-bit cache that they go into (``kv4_append``, ``kv4_load``) and decode attention over it
(``attn_decode_kv4``).  ``run`` computes either the plain form, in elementary torch operations on
32 bits (64 for angles), or calls the package, as ``own`` says.  Head counts, head dims, score
modifiers and the longest contexts are those of ``paper_2510_08726_amd.workloads``; the other sizes
are generic ones: 1 to 64 requests, contexts of 1 to 32768 tokens, pages of 16 to 256 tokens.

The cache is one uint8 tensor [pages, Hkv, page * D * 17 / 16]: for a page and head the codes of K
[page, D / 2] and of V (two E2M1 values a byte, the lower dim in the lower bits), then the scale
bytes of K [D / 32, page] and of V (the exponent plus 127 of a power of two, 255 for NaN).
"""

import math
import random

import torch

own = False

_DTYPE = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
_LIMIT = {"f16": 13, "bf16": 125}      # exponents whose every code is a normal number of the type
_E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _rope(name, op, B, L, Hq, Hkv, D, R, dtype, interleaved, strided, start, factor=1.0):
    return {"name": name, "op": op, "B": B, "L": L, "Hq": Hq, "Hkv": Hkv, "D": D, "R": R, "dtype": dtype,
            "interleaved": interleaved, "strided": strided, "start": start, "factor": factor}


def _slots(name, B, L, page, longest, mix):
    return {"name": name, "op": "slots", "B": B, "L": L, "page": page, "longest": longest, "mix": mix}


def _cache(name, op, B, L, Hkv, D, dtype, page, longest, mix):
    return {"name": name, "op": op, "B": B, "L": L, "Hkv": Hkv, "D": D, "dtype": dtype, "page": page,
            "longest": longest, "mix": mix}


def _decode(name, op, B, Hq, Hkv, D, dtype, page, longest, mix, alibi=False, softcap=0.0, window=0):
    return {"name": name, "op": op, "B": B, "Hq": Hq, "Hkv": Hkv, "D": D, "dtype": dtype, "page": page,
            "longest": longest, "mix": mix, "alibi": alibi, "softcap": softcap, "window": window}


def listed():
    return [
        # The q and k of one decode step of a few requests, deep in their contexts: latency counts.
        _rope("rope decode step", "rope", 8, 1, 32, 8, 128, 128, "bf16", False, False, 20000),
        # A batch of long prompts, read out of the projection's [B, L, H, D], scaled to longer contexts.
        _rope("rope prompts", "rope", 4, 4096, 32, 8, 128, 128, "f16", True, True, 0, 4.0),
        # The gradient in a training step in full precision: half of narrow heads is rotated, odd length.
        _rope("rope gradient", "rope_bwd", 2, 2047, 16, 16, 64, 32, "f32", False, False, 0),
        # The pages and slots of one decode step.
        _slots("slots decode step", 64, 1, 64, 8192, 1),
        # The pages and slots of a batch of prompts of uneven lengths.
        _slots("slots prompts", 256, 2048, 16, 2048, 2),
        # One new token per request goes into the cache, and is read back.
        _cache("cache decode step", "append", 16, 1, 8, 128, "bf16", 64, 4096, 3),
        # Prompts of uneven lengths go into the cache, and are read back.
        _cache("cache prompts", "append", 8, 4095, 8, 128, "f16", 32, 300, 4),
        # A long context is read out for the next piece of its prompt.
        _cache("cache long context", "load", 1, 30001, 8, 128, "bf16", 256, 30001, 0),
        # One request's next token: the smallest decode, latency counts.
        _decode("decode one request", "decode", 1, 32, 8, 128, "bf16", 64, 3001, 0),
        # A batch of requests of uneven lengths, capped scores and a sliding window.
        _decode("decode uneven batch", "decode", 32, 32, 16, 128, "f16", 32, 8192, 5, softcap=50.0, window=4095),
        # Long contexts with grouped heads: the largest decode.
        _decode("decode gqa long", "decode", 16, 32, 8, 128, "bf16", 64, 32768, 0),
        # A whole step of one layer's attention: rotate, append, attend.
        _decode("attention step", "step", 24, 32, 8, 128, "bf16", 64, 6000, 6),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_HEADS = [(32, 32, 128), (32, 8, 128), (64, 8, 128), (32, 16, 128), (16, 16, 64), (12, 12, 64), (32, 4, 64),
          (40, 2, 128)]
_PAGES = [16, 32, 64, 128, 256]


def draw(rng):
    while True:
        op = rng.choice(["rope", "rope", "rope_bwd", "slots", "append", "append", "load", "decode", "decode",
                         "decode", "step"])
        Hq, Hkv, D = rng.choice(_HEADS)
        dtype, page, mix = rng.choice(["f16", "bf16"]), rng.choice(_PAGES), rng.randrange(1 << 20)
        if op in ("rope", "rope_bwd"):
            L = rng.choice([1, _log(rng, 2, 4096)])
            c = _rope("", op, _log(rng, 1, 64), L, Hq, Hkv, D, rng.choice([D, D, D // 2, 24]),
                      rng.choice(["f16", "bf16", "f32"]), rng.random() < 0.5, rng.random() < 0.5,
                      _log(rng, 1, 1 << 20), rng.choice([1.0, 1.0, 8.0]))
        elif op == "slots":
            c = _slots("", _log(rng, 1, 512), rng.choice([1, _log(rng, 2, 2048)]), page, _log(rng, 1, 8192), mix)
        elif op == "append":
            c = _cache("", op, _log(rng, 1, 64), rng.choice([1, _log(rng, 2, 4096)]), Hkv, D, dtype, page,
                       _log(rng, 1, 2048), mix)
        elif op == "load":
            L = _log(rng, 16, 32768)
            c = _cache("", op, _log(rng, 1, 16), L, Hkv, D, dtype, page, L, mix)
        else:
            mod = rng.choice(["plain", "plain", "alibi", "softcap", "window", "softcap window"])
            c = _decode("", op, _log(rng, 1, 64), Hq, Hkv, D, dtype, page, _log(rng, 1, 32768),
                        rng.choice([0, mix]), mod == "alibi", 50.0 if "softcap" in mod else 0.0,
                        _log(rng, 1, 8192) if "window" in mod else 0)
        w = work(c)
        if w["bytes"] <= 5.8e8 and _tokens(c) <= 16 * 32768 * 8 * 128:
            del c["name"]
            return c


def _tokens(c):
    """Cached values (tokens * heads * dims of K) that the plain form spreads out."""
    return 0 if c["op"] in ("rope", "rope_bwd", "slots") else c["B"] * c["longest"] * c["Hkv"] * c["D"]


def _lens(c):
    """Tokens in the cache of each request: all `longest` without a mix, else spread down to one."""
    B, n = c["B"], c["longest"]
    if not c["mix"]:
        return [n] * B
    rng = random.Random(c["mix"])
    return [n] + [_log(rng, 1, n) for _ in range(B - 1)]


def _counts(c):
    """New tokens of each request: one in a decode step, else uneven, some requests without any."""
    if c["L"] == 1:
        return [1] * c["B"]
    rng = random.Random(c["mix"] + 1)
    return [c["L"]] + [rng.randint(0, c["L"]) for _ in range(c["B"] - 1)]


def _pages(n, page):
    return -(-n // page)


def _magnitude(c):
    return 0.1 * math.log(c["factor"]) + 1.0


def _row_bytes(D):
    return D * 17 // 32


def work(c):
    op = c["op"]
    if op in ("rope", "rope_bwd"):
        rows = c["B"] * c["L"] * (c["Hq"] + c["Hkv"])
        size = 4 if c["dtype"] == "f32" else 2
        return {"bytes": 2.0 * rows * c["D"] * size + 4.0 * c["B"] * c["L"] + 4.0 * c["R"],
                "flops": 3.0 * rows * c["R"]}
    if op == "slots":
        new = sum(_pages(n + k, c["page"]) - _pages(n, c["page"]) for n, k in zip(_lens(c), _counts(c)))
        return {"bytes": 12.0 * c["B"] * c["L"] + 12.0 * c["B"] + 8.0 * new, "flops": 0.0}
    if op == "append":     # in, codes out, codes in, out
        n = 2.0 * sum(_counts(c)) * c["Hkv"]
        every = 2.0 * c["B"] * c["L"] * c["Hkv"]
        return {"bytes": n * (2 * c["D"] + 2 * _row_bytes(c["D"])) + every * 2 * c["D"], "flops": 0.0}
    if op == "load":
        n = 2.0 * sum(_lens(c)) * c["Hkv"]
        return {"bytes": n * _row_bytes(c["D"]) + 2.0 * c["B"] * c["L"] * c["Hkv"] * 2 * c["D"], "flops": 0.0}
    seen = sum(min(n, c["window"] or n) for n in _lens(c))
    w = {"bytes": 2.0 * seen * c["Hkv"] * _row_bytes(c["D"]) + 4.0 * c["B"] * c["Hq"] * c["D"],
         "flops": 4.0 * seen * c["Hq"] * c["D"]}
    if op == "step":       # q and k in and out of the rotation, v and k into the cache
        w["bytes"] += c["B"] * c["D"] * (4.0 * c["Hq"] + 8.0 * c["Hkv"])
    return w


# What a program has in hand.

def _normal(shape, dtype, g):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(dtype)


def _heads_first(B, H, L, D, dtype, g, strided):
    """[B, H, L, D]: contiguous, or a view of a projection's [B, L, H, D]."""
    return _normal((B, L, H, D), dtype, g).transpose(1, 2) if strided else _normal((B, H, L, D), dtype, g)


def _frequencies(c):
    """Radians per position of each pair; with a factor, the slow ones are interpolated by parts."""
    R, base = c["R"], 10000.0
    f = base ** (-torch.arange(0, R, 2, dtype=torch.float64, device="cuda") / R)
    if c["factor"] == 1.0:
        return f
    turns = 4096 * f / (2 * math.pi)
    keep = ((turns - 1.0) / (32.0 - 1.0)).clamp(0, 1)
    return f * keep + f / c["factor"] * (1 - keep)


def _spread_pages(c, tokens, g):
    """A table of pages in no order, for the most tokens that any request gets, and the pages left."""
    M = _pages(max(tokens), c["page"]) + 1
    total = c["B"] * M + 3
    perm = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
    return perm[:c["B"] * M].reshape(c["B"], M).contiguous(), perm[c["B"] * M:].contiguous(), total


def _filled(c, table, total, lens, g):
    """A cache of stale bytes with `lens` tokens of each request in it."""
    H, D, P = c["Hkv"], c["D"], c["page"]
    cache = torch.randint(0, 256, (total, H, P * D * 17 // 16), generator=g, device="cuda", dtype=torch.uint8)
    gain = 1.0 + 3.0 * (torch.arange(D, device="cuda") % 13 == 5)     # K has a few strong channels
    for b, n in enumerate(lens):
        if n:
            k = (_normal((1, H, n, D), torch.float32, g) * gain).to(_DTYPE[c["dtype"]])
            v = _normal((1, H, n, D), _DTYPE[c["dtype"]], g)
            _store(cache, k, v, _slots_of(table[b:b + 1], torch.arange(n, device="cuda")[None], P), P, c["dtype"])
    return cache


def _slots_of(table, pos, P):
    return table.long().gather(1, pos // P) * P + pos % P


def prepare(case, seed):
    c = case
    op = c["op"]
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": c}
    if op in ("rope", "rope_bwd"):
        dt = _DTYPE[c["dtype"]]
        s["q"] = _heads_first(c["B"], c["Hq"], c["L"], c["D"], dt, g, c["strided"])
        s["k"] = _heads_first(c["B"], c["Hkv"], c["L"], c["D"], dt, g, c["strided"])
        first = torch.randint(0, c["start"] + 1, (c["B"], 1), generator=g, device="cuda", dtype=torch.int32)
        s["positions"] = (first + torch.arange(c["L"], device="cuda", dtype=torch.int32)).contiguous()
        s["freqs"] = _frequencies(c)
        return s
    lens = _lens(c)
    s["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    if op == "slots":
        counts = _counts(c)
        s["counts"] = torch.tensor(counts, dtype=torch.int32, device="cuda")
        M = _pages(c["longest"] + c["L"], c["page"])
        total = c["B"] * M
        perm = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
        held = [_pages(n, c["page"]) for n in lens]
        s["table"] = perm[:total].reshape(c["B"], M).contiguous()
        need = sum(_pages(n + k, c["page"]) for n, k in zip(lens, counts)) - sum(held)
        need = need * 9 // 10 if c["mix"] % 5 == 2 else need + 7      # now and then too few are left
        s["free"] = torch.randperm(max(need, 1), generator=g, device="cuda").to(torch.int32)
        return s
    if op == "append":
        counts = _counts(c)
        tokens = [n + k for n, k in zip(lens, counts)]
        s["table"], _, total = _spread_pages(c, tokens, g)
        s["cache"] = torch.randint(0, 256, (total, c["Hkv"], c["page"] * c["D"] * 17 // 16), generator=g,
                                   device="cuda", dtype=torch.uint8)
        s["k"] = _normal((c["B"], c["Hkv"], c["L"], c["D"]), _DTYPE[c["dtype"]], g)
        s["v"] = _normal((c["B"], c["Hkv"], c["L"], c["D"]), _DTYPE[c["dtype"]], g)
        l = torch.arange(c["L"], device="cuda")[None]
        n = torch.tensor(counts, device="cuda")[:, None]
        at = _slots_of(s["table"], s["lens"].long()[:, None] + torch.minimum(l, (n - 1).clamp(min=0)), c["page"])
        s["slots"] = torch.where(l < n, at, -1).contiguous()
        s["ends"] = torch.tensor(tokens, dtype=torch.int32, device="cuda")
        return s
    s["table"], _, total = _spread_pages(c, lens, g)
    s["cache"] = _filled(c, s["table"], total, lens, g)
    if op == "load":
        return s
    s["q"] = _normal((c["B"], c["Hq"], 1, c["D"]), _DTYPE[c["dtype"]], g)
    s["slopes"] = None
    if c["alibi"]:
        s["slopes"] = 2.0 ** (-8.0 * torch.arange(1, c["Hq"] + 1, device="cuda", dtype=torch.float32) / c["Hq"])
    if op == "step":       # the last token of each request is the step's
        s["k"] = _normal((c["B"], c["Hkv"], 1, c["D"]), _DTYPE[c["dtype"]], g)
        s["v"] = _normal((c["B"], c["Hkv"], 1, c["D"]), _DTYPE[c["dtype"]], g)
        s["freqs"] = 10000.0 ** (-torch.arange(0, c["D"], 2, dtype=torch.float64, device="cuda") / c["D"])
        s["positions"] = (s["lens"] - 1)[:, None].contiguous()
        s["slots"] = _slots_of(s["table"], s["positions"].long(), c["page"])
    return s


# Plain forms.

def _rotate(x, positions, freqs, interleaved, magnitude, sign):
    R = 2 * freqs.numel()
    t = positions.double()[:, None, :, None] * freqs
    co, si = (t.cos() * magnitude).float(), (t.sin() * (sign * magnitude)).float()
    y = x.float()
    if interleaved:
        a, b = y[..., 0:R:2], y[..., 1:R:2]
        r = torch.stack((a * co - b * si, a * si + b * co), -1).flatten(-2)
    else:
        a, b = y[..., :R // 2], y[..., R // 2:R]
        r = torch.cat((a * co - b * si, a * si + b * co), -1)
    return torch.cat((r, y[..., R:]), -1).to(x.dtype)


def _place(lens, counts, table, free, P, L):
    M, F = table.shape[1], free.numel()
    n, k = lens.long(), counts.long()
    held = (n + P - 1) // P
    need = ((torch.minimum(n + k, torch.full_like(n, M * P)) + P - 1) // P - held).clamp(min=0)
    start = need.cumsum(0) - need
    got = torch.minimum((F - start).clamp(min=0), need)
    stored = torch.minimum((held + got) * P - n, k).clamp(min=0)
    col = torch.arange(M, device=table.device)[None]
    new = (col >= held[:, None]) & (col < (held + got)[:, None])
    pick = (start[:, None] + col - held[:, None]).clamp(0, max(F - 1, 0))
    out = torch.where(new, free[pick], table)
    pos = n[:, None] + torch.arange(L, device=table.device)[None]
    at = _slots_of(out, pos.clamp(max=M * P - 1), P)
    keep = torch.arange(L, device=table.device)[None] < stored[:, None]
    return torch.where(keep, at, -1), pos.to(torch.int32), (n + stored).to(torch.int32), \
        got.sum().to(torch.int32).reshape(1), out


def _quantise(x, dtype):
    """x [N, H, D] -> codes [N, H, D / 2], scale bytes [N, H, D / 32]."""
    N, H, D = x.shape
    y = x.float().reshape(N, H, D // 32, 32)
    fine = y.isfinite().all(-1)
    y = torch.where(fine[..., None], y, 0.0)
    e = ((y.abs().amax(-1).view(torch.int32) + 0x1FFFFF) >> 23) - 129
    e = e.clamp(-_LIMIT[dtype], _LIMIT[dtype])
    z = y * ((127 - e) << 23).view(torch.float32)[..., None]
    a = z.abs()
    c = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0))
    c = (c + 8 * (z < 0)).to(torch.uint8).reshape(N, H, D)
    return c[..., 0::2] | (c[..., 1::2] << 4), torch.where(fine, e + 127, 255).to(torch.uint8)


def _parts(cache, P, D):
    """Views of a cache: codes of K and V [pages, H, P, D / 2], scales of K and V [pages, H, D / 32, P]."""
    n, H, code, scale = cache.shape[0], cache.shape[1], P * D // 2, P * D // 32
    x = cache.split([code, code, scale, scale], -1)
    return [t.unflatten(-1, (P, D // 2)) for t in x[:2]] + [t.unflatten(-1, (D // 32, P)) for t in x[2:]]


def _store(cache, k, v, slots, P, dtype):
    D = k.shape[-1]
    keep = slots.reshape(-1) >= 0
    at = slots.reshape(-1)[keep]
    kc, vc, ks, vs = _parts(cache, P, D)
    rows = lambda x: x.transpose(1, 2).flatten(0, 1)[keep]     # noqa: E731  [tokens, H, D]
    kc[at // P, :, at % P], ks[at // P, :, :, at % P] = _quantise(rows(k), dtype)
    vc[at // P, :, at % P], vs[at // P, :, :, at % P] = _quantise(rows(v), dtype)


def _values(codes, scales):
    """codes [..., P, D / 2], scales [..., D / 32, P] -> values [..., P, D] in 32 bits."""
    pair = torch.tensor(_E2M1 + tuple(-x for x in _E2M1), device=codes.device)
    lut = torch.stack((pair.repeat(16), pair.repeat_interleave(16)), -1)       # byte -> its two values
    x = lut[codes.int()].flatten(-2).unflatten(-1, (-1, 32))
    s = torch.where(scales == 255, float("nan"), torch.ldexp(torch.ones((), device=codes.device), scales.int() - 127))
    return (x * s.transpose(-1, -2)[..., None]).flatten(-2)


def _gather(cache, table, P, D):
    """K and V of every page of the table in 32 bits, [B, H, M P, D]."""
    kc, vc, ks, vs = (t[table.long()].transpose(1, 2) for t in _parts(cache, P, D))    # [B, H, M, ...]
    return _values(kc, ks).flatten(2, 3), _values(vc, vs).flatten(2, 3)


def _load(cache, table, starts, ends, L, P, D, dtype):
    k, v = _gather(cache, table, P, D)
    pos = starts.long()[:, None] + torch.arange(L, device=cache.device)[None]
    there = (pos < ends.long()[:, None]) & (pos < k.shape[2])
    at = pos.clamp(max=k.shape[2] - 1)[:, None, :, None].expand(-1, k.shape[1], -1, D)
    return [torch.where(there[:, None, :, None], t.gather(2, at), 0.0).to(dtype) for t in (k, v)]


def _attend(q, cache, table, lens, slopes, c):
    P, D, G = c["page"], c["D"], c["Hq"] // c["Hkv"]
    k, v = _gather(cache, table, P, D)
    B, H, N, _ = k.shape
    j = torch.arange(N, device=q.device)[None]
    n = lens.long()[:, None]
    seen = (j < n) & (j >= n - (c["window"] or N + 1))
    k, v = (torch.where(seen[:, None, :, None], t, 0.0) for t in (k, v))
    x = (q.float().reshape(B, H, G, D) @ k.transpose(2, 3)) * D ** -0.5
    if c["softcap"]:
        x = c["softcap"] * torch.tanh(x / c["softcap"])
    if slopes is not None:
        x = x + slopes.reshape(1, H, G, 1) * (j - (n - 1)).float()[:, None, None]
    x = torch.where(seen[:, None, None], x, -math.inf)
    top = x.amax(-1, keepdim=True)
    w = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
    total = w.sum(-1, keepdim=True)
    o = torch.where(total > 0, (w @ v) / total, 0.0)
    return o.reshape(B, H * G, 1, D).to(q.dtype)


def run(state):
    s, c = state, state["case"]
    op = c["op"]
    if own:
        return _run_own(s, c, op)
    if op in ("rope", "rope_bwd"):
        sign = 1.0 if op == "rope" else -1.0
        return [_rotate(s[t], s["positions"], s["freqs"], c["interleaved"], _magnitude(c), sign) for t in ("q", "k")]
    if op == "slots":
        return _place(s["lens"], s["counts"], s["table"], s["free"], c["page"], c["L"])
    if op == "append":
        _store(s["cache"], s["k"], s["v"], s["slots"], c["page"], c["dtype"])
        return _load(s["cache"], s["table"], s["lens"], s["ends"], c["L"], c["page"], c["D"], _DTYPE[c["dtype"]])
    if op == "load":
        return _load(s["cache"], s["table"], torch.zeros_like(s["lens"]), s["lens"], c["L"], c["page"], c["D"],
                     _DTYPE[c["dtype"]])
    q = s["q"]
    if op == "step":
        q, k = (_rotate(t, s["positions"], s["freqs"], False, 1.0, 1.0) for t in (q, s["k"]))
        _store(s["cache"], k, s["v"], s["slots"], c["page"], c["dtype"])
        return _attend(q, s["cache"], s["table"], s["lens"], s["slopes"], c), q, k
    return _attend(q, s["cache"], s["table"], s["lens"], s["slopes"], c)


def _run_own(s, c, op):
    import paper_2510_08726_amd as pa
    if op == "rope":
        return pa.rope_fwd(s["q"], s["k"], s["positions"], s["freqs"], interleaved=c["interleaved"],
                           magnitude=_magnitude(c))
    if op == "rope_bwd":
        return pa.rope_bwd(s["q"], s["k"], s["positions"], s["freqs"], interleaved=c["interleaved"],
                           magnitude=_magnitude(c))
    if op == "slots":
        return (*pa.kv_slots(s["lens"], s["counts"], s["table"], s["free"], c["page"], c["L"]), s["table"])
    if op == "append":
        pa.kv4_append(s["k"], s["v"], s["cache"], s["slots"])
        return pa.kv4_load(s["cache"], s["table"], s["ends"], c["L"], c["D"], _DTYPE[c["dtype"]], starts=s["lens"])
    if op == "load":
        return pa.kv4_load(s["cache"], s["table"], s["lens"], c["L"], c["D"], _DTYPE[c["dtype"]])
    q, k = s["q"], None
    if op == "step":
        q, k = pa.rope_fwd(q, s["k"], s["positions"], s["freqs"])
        pa.kv4_append(k, s["v"], s["cache"], s["slots"])
    o = pa.attn_decode_kv4(q, s["cache"], s["table"], s["lens"], alibi_slopes=s["slopes"],
                           softcap=c["softcap"] or None, window=c["window"] or None)
    return (o, q, k) if op == "step" else o


# The definitions in 64 bits, apart from the plain forms.

def _rotation64(x, positions, freqs, interleaved, magnitude, sign):
    R = 2 * freqs.numel()
    y = x.double().clone()
    z = x.double()[..., :R]
    pairs = z.unflatten(-1, (R // 2, 2)) if interleaved else z.unflatten(-1, (2, R // 2)).transpose(-1, -2)
    turn = torch.polar(torch.full((), magnitude, dtype=torch.float64, device=x.device),
                       sign * positions.double()[:, None, :, None] * freqs)
    r = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
    y[..., :R] = r.flatten(-2) if interleaved else r.transpose(-1, -2).flatten(-2)
    return y


def _held64(x, dtype):
    """The values that the 4-bit form of x [..., D] stands for: the nearest of 15 multiples of 2^e."""
    y = x.double().unflatten(-1, (-1, 32))
    top = y.abs().amax(-1, keepdim=True)
    # 4 <= top / 2^e <= 7 or 3.5 < top / 2^e < 4; frexp: top = m 2^q, 1/2 <= m < 1
    m, q = torch.frexp(top)
    e = torch.where(top > 0, q - 3 + (m > 0.875).int(), -1000).clamp(-_LIMIT[dtype], _LIMIT[dtype])
    z = torch.ldexp(y.abs(), -e)
    step = torch.where(z < 2, 0.5, torch.where(z < 4, 1.0, 2.0)).double()     # of the code's binade; ties to even
    near = (torch.round(z / step) * step).clamp(max=6.0)
    near = torch.where(z < 1, torch.round(2 * z) / 2, near)
    return (torch.ldexp(near, e) * y.sign()).flatten(-2)


def _context64(cache, row, n, P, D):
    """K and V of the first n tokens of one request, [H, n, D]."""
    pages = row[:_pages(n, P)].long()
    raw = cache[pages].long()                                                 # [pages, H, bytes]
    half, few = P * D // 2, P * D // 32
    out = []
    for code, scale in ((raw[..., :half], raw[..., 2 * half:2 * half + few]),
                        (raw[..., half:2 * half], raw[..., 2 * half + few:])):
        nib = torch.stack((code & 15, code >> 4), -1).reshape(len(pages), -1, P, D)
        mag = nib & 7
        man, ex = mag & 1, mag >> 1
        x = torch.where(ex == 0, 0.5 * man, torch.ldexp(1.0 + 0.5 * man.double(), ex - 1))
        x = torch.where(nib >= 8, -x, x)
        s = torch.ldexp(torch.ones((), dtype=torch.float64, device=cache.device), scale - 127)
        x = x * s.reshape(len(pages), -1, D // 32, P).transpose(2, 3).repeat_interleave(32, -1)
        out.append(x.transpose(0, 1).reshape(-1, len(pages) * P, D)[:, :n])
    return out


def exact(case, seed):
    c = case
    op = c["op"]
    if op == "slots":
        return None
    s = prepare(case, seed)
    if op in ("rope", "rope_bwd"):
        sign = 1.0 if op == "rope" else -1.0
        return [_rotation64(s[t], s["positions"], s["freqs"], c["interleaved"], _magnitude(c), sign)
                for t in ("q", "k")]
    if op == "append":
        there = (s["slots"] >= 0)[:, None, :, None]
        return [torch.where(there, _held64(s[t], c["dtype"]), 0.0) for t in ("k", "v")]
    if op == "load":
        out = [torch.zeros(c["B"], c["Hkv"], c["L"], c["D"], dtype=torch.float64, device="cuda") for _ in range(2)]
        for b, n in enumerate(_lens(c)):
            for o, x in zip(out, _context64(s["cache"], s["table"][b], n, c["page"], c["D"])):
                o[b, :, :n] = x
        return out
    q = s["q"].double()
    if op == "step":
        one = lambda x: _rotation64(x, s["positions"], s["freqs"], False, 1.0, 1.0)     # noqa: E731
        turned = one(s["q"]), one(s["k"])
        q = turned[0].to(s["q"].dtype).double()
        new_k, new_v = _held64(turned[1].to(s["k"].dtype), c["dtype"]), _held64(s["v"], c["dtype"])
    G = c["Hq"] // c["Hkv"]
    out = torch.zeros_like(q)
    for b, n in enumerate(_lens(c)):
        k, v = _context64(s["cache"], s["table"][b], n, c["page"], c["D"])
        if op == "step":
            k, v = k.clone(), v.clone()
            k[:, -1], v[:, -1] = new_k[b, :, 0], new_v[b, :, 0]
        lo = max(0, n - c["window"]) if c["window"] else 0
        x = torch.matmul(q[b, :, 0].reshape(c["Hkv"], G, -1), k[:, lo:].transpose(1, 2).contiguous())
        x = x / math.sqrt(c["D"])
        if c["softcap"]:
            x = torch.tanh(x / c["softcap"]) * c["softcap"]
        if s["slopes"] is not None:
            far = torch.arange(lo - n + 1, 1, device="cuda", dtype=torch.float64)
            x = x + s["slopes"].double().reshape(c["Hkv"], G, 1) * far
        out[b, :, 0] = torch.matmul(torch.softmax(x, -1), v[:, lo:].contiguous()).reshape(c["Hq"], -1)
    return (out, *turned) if op == "step" else out
