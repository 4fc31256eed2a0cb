"""The error that attention's outputs have by the roundings that its kernels choose, and no other: what a test of the kernels may
compare theirs with.

``emulate`` computes in float64 and rounds where attn_bwd.h says: the weights of O to the type of Q (their sum not),
O, the log-sum-exp to fp32, P to the type for dV, dS to the type for dK and as two values of it for dQ, and each
gradient.  Sums in fp32, scores and exponentials are off by 2^-20 of what they are made of at most
(train_cases.bounds): against the smallest of the roundings above, 2^-12 in fp16, whose root mean square is 2^-12 /
sqrt(3), a term that adds less than a fiftieth to a root mean square.  So ``check`` allows a tenth more than the emulated error;
a rounding too many, or bits too few, cost more (test_train_errors.py)."""

import numpy as np
import torch

from oracle import train
from train_cases import DT

MORE = 1.1
# (B, Hq, Hkv, Lq, Lk, D, causal, slopes, softcap, window)
CASES = [
    (1, 4, 2, 300, 300, 128, True, None, None, None),
    (1, 2, 1, 260, 500, 64, False, None, None, None),
    (1, 4, 2, 300, 300, 64, True, None, 30.0, 100),
    (2, 4, 4, 200, 333, 128, True, (0.5, 0.25, 0.0625, 0.01), None, None),
]
# Biases that make the log-sum-exp of a row as large as the distance of its farthest key: thousands.
FAR = [
    (1, 2, 1, 8192, 300, 128, False, (0.84, 0.25), None, None),
    (1, 2, 2, 8192, 150, 64, False, (0.84, 0.25), None, None),
    (1, 2, 2, 40, 8192, 64, False, (-0.84, -0.25), None, None),
    (1, 2, 1, 2500, 2500, 64, True, (-0.84, -0.25), None, None),
    (1, 2, 2, 2100, 2500, 128, True, (-0.84, -0.25), None, 1700),
]


def to(x, dtype):
    return torch.from_numpy(np.ascontiguousarray(x)).to(dtype).double().numpy()


def emulate(do, q, k, v, dtype, *, scale, causal=False, alibi_slopes=None, softcap=None, window=None, dq_once=False, drop=0,
            exponent=0.0):
    """o, lse, dq, dk, dv with the kernels' roundings.  For mutants: dS for dQ rounded once, `drop` bits less of dS, and exponents off
    by up to `exponent`."""
    T, half = DT[dtype], dtype == "f16"
    B, Hq, Lq, D = q.shape
    Hkv = k.shape[1]
    G = Hq // Hkv
    shift = 2.0 ** 15 if half else 1.0
    noise = np.random.default_rng(1)
    r = {n: np.zeros(t.shape) for n, t in (("o", q), ("dq", q), ("dk", k), ("dv", v))}
    r["lse"] = np.full(q.shape[:3], -np.inf)
    for b in range(B):
        for h in range(Hq):
            kh = h // G
            s, d, seen = train.scores(q[b, h], k[b, kh], scale=scale, causal=causal, slope=None if alibi_slopes is None else alibi_slopes[h],
                                      softcap=softcap, window=window)
            some = seen.any(-1)
            top = np.where(some, s.max(-1, initial=-np.inf), 0.0)
            e = np.where(seen, np.exp(s - top[:, None]), 0.0)
            total = np.where(some, e.sum(-1), 1.0)
            o = to((to(e, T) @ v[b, kh]) / total[:, None], T)
            lse = np.where(some, top + np.log(total), -np.inf)
            r["o"][b, h], r["lse"][b, h] = o, to(lse, torch.float32)
            known = np.where(some, r["lse"][b, h], 0.0)
            P = np.where(seen, np.exp(np.where(seen, s, 0.0) - known[:, None] + exponent * noise.uniform(-1, 1, s.shape)), 0.0)
            g = np.where(some[:, None], do[b, h], 0.0)
            dS = P * (g @ v[b, kh].T - (g * o).sum(-1, keepdims=True)) * d
            norm = lambda t: np.sqrt((t ** 2).sum(-1).max())     # noqa: E731
            up = 2.0 ** (14 - np.frexp(2.02 * norm(do[b, kh * G:(kh + 1) * G]) * norm(v[b, kh]))[1]) if half else 1.0
            held = dS * up
            first = to(held, T)
            if drop:
                m, x = np.frexp(held)
                bits = {"f16": 11, "bf16": 8}[dtype] - drop
                first = np.ldexp(np.round(m * 2 ** bits) / 2 ** bits, x)
            both = first if dq_once or drop else first + to(held - first, T)
            r["dv"][b, kh] += (to(P * shift, T) / shift).T @ g
            r["dk"][b, kh] += (first / up).T @ q[b, h] * scale
            r["dq"][b, h] = to((both / up) @ k[b, kh] * scale, T)
    r["dk"], r["dv"] = to(r["dk"], T), to(r["dv"], T)
    return r


def rms(a, b):
    blind = ~np.isfinite(b)
    assert np.array_equal(a[blind], b[blind])
    return float(np.sqrt(np.mean(np.where(blind, 0.0, a - np.where(blind, 0.0, b)) ** 2)))


def shares(got, want, emulated):
    """Each output's root mean square error over the emulated one."""
    return {n: rms(t, want[n]) / max(rms(emulated[n], want[n]), 1e-300) for n, t in got.items()}


def inputs(case, dtype):
    """Host tensors do, q, k, v, slopes of a case."""
    B, Hq, Hkv, Lq, Lk, D, _, slopes, _, _ = case
    g = torch.Generator().manual_seed(sum(case[:6]))
    t = lambda H, L: torch.randn((B, H, L, D), generator=g).to(DT[dtype])     # noqa: E731
    return t(Hq, Lq), t(Hq, Lq), t(Hkv, Lk), t(Hkv, Lk), None if slopes is None else torch.tensor(slopes, dtype=torch.float32)


def both64(case, x, dtype, **mutant):
    """The definition in 64 bits, and the emulated outputs."""
    do, q, k, v, slopes = x
    how = dict(scale=q.shape[3] ** -0.5, causal=case[6], softcap=case[8], window=case[9],
               alibi_slopes=None if slopes is None else slopes.double().numpy())
    x = [t.double().numpy() for t in (do, q, k, v)]
    return train.attention_grad(*x, **how), emulate(*x, dtype, **how, **mutant)
