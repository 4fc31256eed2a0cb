"""Rotary positions and the paged 4-bit cache, in float64 — TEST INFRASTRUCTURE ONLY.

Plain definitions of what ``include/rope.h`` and ``include/kv4.h`` state, with
loops over requests and no code shared with the GPU path:

* ``rope``: each pair of dims is turned by position * frequency;
* ``held``: the codes, scale bytes and values of the 4-bit form, by trying every code;
* ``pack`` / ``unpack``: the cache's bytes, one token and head at a time;
* ``slots``: pages and slots of new tokens, one token at a time;
* ``decode``: ``oracle.attention`` of each request over its own tokens.
"""

import math

import numpy as np

from .attention import attention

VALUES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
LIMIT = {"f16": 13, "bf16": 125}


def rope(x, positions, freqs, *, interleaved=False, magnitude=1.0, transpose=False):
    """x [B, H, L, D], positions [B, L], freqs [R / 2] -> the rotated x."""
    x = np.asarray(x, dtype=np.float64)
    y = x.copy()
    n = len(freqs)
    for i in range(n):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + n)
        t = np.asarray(positions, dtype=np.longdouble) * np.longdouble(freqs[i])
        c = (magnitude * np.cos(t)).astype(np.float64)[:, None, :]
        s = (magnitude * np.sin(t)).astype(np.float64)[:, None, :]
        if transpose:
            s = -s
        y[..., a] = c * x[..., a] - s * x[..., b]
        y[..., b] = s * x[..., a] + c * x[..., b]
    return y


def frequencies(R, base, scaling=None, factor=1.0, original_length=0, slow=1.0, fast=32.0):
    out = []
    for i in range(R // 2):
        b = base * factor ** (R / (R - 2)) if scaling == "base" else base
        f = b ** (-2 * i / R)
        if scaling == "linear":
            f = f / factor
        if scaling == "parts":
            turns = original_length * f / (2 * math.pi)
            w = min(max((turns - slow) / (fast - slow), 0.0), 1.0)
            f = w * f + (1 - w) * f / factor
        out.append(f)
    return np.array(out)


def held(x, dtype):
    """x [..., D] -> codes [..., D] (0 .. 15), scale bytes [..., D / 32], values [..., D]."""
    x = np.asarray(x, dtype=np.float64)
    y = x.reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    fine = np.isfinite(y).all(-1)
    y = np.where(fine[..., None], y, 0.0)
    top = np.abs(y).max(-1)
    e = np.full(top.shape, -LIMIT[dtype])
    for k in range(-LIMIT[dtype] + 1, LIMIT[dtype] + 1):       # the smallest e with top <= 7 * 2^e
        e = np.where(top > 7.0 * 2.0 ** (k - 1), k, e)
    z = np.abs(y) / np.exp2(e)[..., None]
    best, code = np.full(z.shape, np.inf), np.zeros(z.shape, dtype=np.int64)
    for c in (0, 2, 4, 6, 1, 3, 5, 7):                         # even codes first: they keep a tie
        d = np.abs(z - VALUES[c])
        code = np.where(d < best, c, code)
        best = np.minimum(d, best)
    values = np.where(fine[..., None], np.copysign(VALUES[code], y) * np.exp2(e)[..., None], np.nan)
    code = np.where(fine[..., None], code + 8 * np.signbit(y), 0)
    return code.reshape(x.shape), np.where(fine, e + 127, 255), values.reshape(x.shape)


def page_bytes(page, D):
    return 2 * (page * D // 2 + page * D // 32)


def pack(cache, slot, h, code_k, scale_k, code_v, scale_v, page, D):
    """Write one token of one head into cache [pages, H, bytes]."""
    row = slot % page
    to = cache[slot // page, h]
    half, few = page * D // 2, page * D // 32
    for k, (code, scale) in enumerate(((code_k, scale_k), (code_v, scale_v))):
        to[k * half + row * D // 2:k * half + (row + 1) * D // 2] = code[0::2] + 16 * code[1::2]
        for j in range(D // 32):
            to[2 * half + k * few + j * page + row] = scale[j]


def unpack(cache, slot, h, page, D):
    """Values of K and V of one token of one head."""
    row = slot % page
    at = cache[slot // page, h].astype(np.int64)
    half, few = page * D // 2, page * D // 32
    out = []
    for k in range(2):
        b = at[k * half + row * D // 2:k * half + (row + 1) * D // 2]
        code = np.stack([b & 15, b >> 4], -1).reshape(-1)
        x = np.where(code & 8, -1.0, 1.0) * VALUES[code & 7]
        s = at[2 * half + k * few + row::page][:D // 32]
        out.append(x * np.repeat(np.where(s == 255, np.nan, np.exp2(s - 127.0)), 32))
    return out


def slots(lens, counts, table, free, page, L):
    """One token at a time: (slots, positions, new lengths, pages taken, table)."""
    table = np.array(table)
    B, M = table.shape
    out = np.full((B, L), -1, dtype=np.int64)
    pos = np.zeros((B, L), dtype=np.int64)
    new, taken = [], 0
    for b in range(B):
        n = min(max(int(lens[b]), 0), M * page)
        pos[b] = n + np.arange(L)
        for l in range(min(int(counts[b]), L)):
            if n == M * page:
                break
            if n % page == 0:
                if taken == len(free):
                    break
                table[b, n // page] = free[taken]
                taken += 1
            out[b, l] = int(table[b, n // page]) * page + n % page
            n += 1
        new.append(n)
    return out, pos, np.array(new), taken, table


def decode(q, ks, vs, *, scale, slopes=None, softcap=None, window=None):
    """q [B, Hq, 1, D]; ks, vs: for each request [Hkv, n, D] (n may be 0).  Returns the
    output and, for tolerances, the weighted mean of |v|."""
    out, mean = np.zeros(q.shape), np.zeros(q.shape)
    for b, (k, v) in enumerate(zip(ks, vs)):
        if k.shape[1]:
            kw = dict(scale=scale, causal=True, alibi_slopes=slopes, softcap=softcap, window=window)
            out[b] = attention(q[b:b + 1], k[None], v[None], **kw)[0]
            mean[b] = attention(q[b:b + 1], k[None], np.abs(v[None]), **kw)[0]
    return out, mean
