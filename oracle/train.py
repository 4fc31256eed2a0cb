"""Attention's forward pass with its rows' log-sum-exp, and its gradients, in float64.

The definitions of ``include/attn_bwd.h`` written out over whole score matrices, head by head:
s = mod(scale q k^T) + bias with masked entries -inf, lse = log sum exp(s), P = exp(s - lse), and the
derivative of O = P v by the chain rule.  Nothing here is shared with the kernels: the
inputs are host arrays, everything is numpy.
"""

import numpy as np


def scores(q, k, *, scale, causal, slope, softcap, window):
    """(s, mod', visible) of one head, [Lq, Lk] each."""
    Lq, Lk = len(q), len(k)
    x = scale * (q @ k.T)
    d = np.ones_like(x)
    if softcap:
        t = np.tanh(x / softcap)
        x, d = softcap * t, 1.0 - t * t
    ahead = (np.arange(Lq)[:, None] + (Lk - Lq)) - np.arange(Lk)[None]
    if slope is not None:
        x = x - slope * ahead
    seen = np.ones((Lq, Lk), dtype=bool)
    if causal:
        seen = ahead >= 0
        if window:
            seen &= ahead < window
    return np.where(seen, x, -np.inf), d, seen


def attention_grad(do, q, k, v, *, scale, causal=False, alibi_slopes=None, softcap=None, window=None):
    """o, lse, dq, dk, dv, and the sums of magnitudes behind each gradient, for error bounds:

    what a relative error of every P (``dv_abs``) or dS (``dq_abs``, ``dk_abs``) costs at most, and what an absolute
    error of delta_i of sum_d |do| (|o| + P |v|) costs (``dq_delta``, ``dk_delta``); what an absolute error of every P
    costs (``dv_each``) and one of every dS of |do| |v| of the KV head's largest rows (``dq_each``, ``dk_each``); ``reach``
    is the largest sum_d |scale q_d k_d| of a row."""
    B, Hq, Lq, D = q.shape
    Hkv, Lk = k.shape[1], k.shape[2]
    G = Hq // Hkv
    r = {n: np.zeros(q.shape) for n in ("o", "o_abs", "dq", "dq_abs", "dq_delta", "dq_each")}
    r.update({n: np.zeros(k.shape) for n in ("dk", "dk_abs", "dk_delta", "dk_each", "dv", "dv_abs", "dv_each")})
    r["lse"], r["reach"] = np.full(q.shape[:3], -np.inf), np.zeros(q.shape[:3])
    for b in range(B):
        for h in range(Hq):
            kh = h // G
            qq, kk, vv, g = q[b, h], k[b, kh], v[b, kh], do[b, h]
            slope = None if alibi_slopes is None else alibi_slopes[h]
            s, d, seen = scores(qq, kk, scale=scale, causal=causal, slope=slope, softcap=softcap, window=window)
            some = seen.any(-1)
            top = np.where(some, s.max(-1, initial=-np.inf), 0.0)
            e = np.where(seen, np.exp(s - top[:, None]), 0.0)
            total = e.sum(-1)
            P = np.divide(e, total[:, None], out=np.zeros_like(e), where=total[:, None] > 0)
            r["lse"][b, h] = np.where(some, top + np.log(np.where(some, total, 1.0)), -np.inf)
            r["reach"][b, h] = abs(scale) * (np.abs(qq) @ np.abs(kk).T).max(-1)
            r["o"][b, h], r["o_abs"][b, h] = P @ vv, P @ np.abs(vv)
            g = np.where(some[:, None], g, 0.0)
            dP = g @ vv.T
            dS = P * (dP - (P * dP).sum(-1, keepdims=True)) * d * scale
            off = P * (np.abs(g) * (np.abs(r["o"][b, h]) + r["o_abs"][b, h])).sum(-1, keepdims=True) * d * abs(scale)
            r["dv"][b, kh] += P.T @ g
            r["dv_abs"][b, kh] += P.T @ np.abs(g)
            r["dq"][b, h], r["dq_abs"][b, h], r["dq_delta"][b, h] = dS @ kk, np.abs(dS) @ np.abs(kk), off @ np.abs(kk)
            r["dk"][b, kh] += dS.T @ qq
            r["dk_abs"][b, kh] += np.abs(dS).T @ np.abs(qq)
            r["dk_delta"][b, kh] += off.T @ np.abs(qq)
            most = lambda t: np.sqrt((np.where(np.isfinite(t), t, 0.0) ** 2).sum(-1).max())     # noqa: E731
            size = abs(scale) * most(do[b, kh * G:(kh + 1) * G]) * most(v[b, kh])
            r["dv_each"][b, kh] += np.abs(g).sum(0)
            r["dq_each"][b, h] += size * np.abs(kk).sum(0)
            r["dk_each"][b, kh] += size * np.abs(qq).sum(0)
    return r


def rmsnorm(h, weight, eps, offset):
    """y and rstd of rows h [N, M] in float64 (weight None: ones, without the offset)."""
    rstd = 1.0 / np.sqrt((h * h).mean(-1) + eps)
    return h * rstd[:, None] * (1.0 if weight is None else weight + offset), rstd


def rmsnorm_grad(dy, h, rstd, weight, dh, offset):
    """dx and dweight, and their sums of magnitudes: (dx, dw, of dx's terms, of the mean behind dx, of dw)."""
    n = h * rstd[:, None]
    g = dy * (1.0 if weight is None else weight + offset)
    mean, size = (g * n).mean(-1, keepdims=True), np.abs(g * n).mean(-1, keepdims=True)
    r = rstd[:, None]
    d = r * (g - n * mean) + (0.0 if dh is None else dh)
    terms = r * (np.abs(g) + np.abs(n * mean)) + (0.0 if dh is None else np.abs(dh))
    return d, (dy * n).sum(0), terms, r * np.abs(n) * size, np.abs(dy * n).sum(0)


def codes8(y, code, group):
    """The values of the codes nearest to y / scale (ties to even), and the scales in fp32: y [N, M] in groups."""
    N, M = y.shape
    step = group or M
    values, scales = np.zeros_like(y), []
    if code == "int8":
        grid = np.arange(128.0)
    else:     # 4 bits of exponent (bias 7), 3 of mantissa
        grid = np.array([(m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)) for e in range(16) for m in range(8)][:127])
    for a in range(0, M, step):
        part = y[:, a:a + step]
        with np.errstate(invalid="ignore", over="ignore"):
            s = (np.abs(part).max(-1) / grid[-1]).astype(np.float32)
        s = np.where(np.isfinite(s), s, np.float32(np.nan))
        scales.append(s)
        fine = np.isfinite(s) & (s > 0)
        z = np.where(fine[:, None], np.abs(part) / np.where(fine, s, 1.0).astype(np.float64)[:, None], 0.0)
        hi = np.clip(np.searchsorted(grid, z), 1, len(grid) - 1)
        lo = hi - 1
        below, above = z - grid[lo], grid[hi] - z
        at = np.where((below < above) | ((below == above) & (lo % 2 == 0)), lo, hi)
        values[:, a:a + step] = grid[at] * np.where(fine[:, None], np.sign(part), 0.0)
    return values, np.stack(scales, -1)
