"""Inputs of the tests of attention in training, and the error bounds of its outputs."""

import math

import numpy as np
import torch

from oracle import train

DT = {"f16": torch.float16, "bf16": torch.bfloat16}


def draw(B, Hq, Hkv, Lq, Lk, D, dtype, seed, alibi=False, size=1.0):
    """Host tensors do, q, k, v and slopes (or None): N(0, 1), k with a few strong dims, do times `size`."""
    g = torch.Generator().manual_seed(seed)
    t = lambda H, L: torch.randn((B, H, L, D), generator=g)     # noqa: E731
    q, k, v, do = t(Hq, Lq), t(Hkv, Lk) * (1.0 + 2.0 * (torch.arange(D) % 13 == 5)), t(Hkv, Lk), size * t(Hq, Lq)
    slopes = None
    if alibi:
        slopes = torch.tensor([2.0 ** (-8.0 * (h + 1) / Hq) for h in range(Hq)], dtype=torch.float32)
    return [x.to(DT[dtype]) for x in (do, q, k, v)] + [slopes]


def oracle64(do, q, k, v, slopes, **how):
    x = [t.double().numpy() for t in (do, q, k, v)]
    how["scale"] = 1.0 / math.sqrt(q.shape[3]) if how.get("scale") is None else how["scale"]
    return train.attention_grad(*x, alibi_slopes=None if slopes is None else slopes.double().numpy(), **how)


def bounds(r, dtype, slopes=None, softcap=None, Lk=0):
    """The most that each output may be off.

    u = eps / 2 of the type is one rounding.  A score is a sum of at most 128 products in fp32
    (chained 16 at a time) and one multiplication: under 2^-20 of its sum of magnitudes; its exponent is
    formed with lse, three roundings of 2^-24 of |s|, |lse| and the bias; the cap is off by 2^-21 of itself.  A
    weight's relative error is the error of its exponent (e) and 2^-20 for the exponential.  P and dS are rounded once
    (u), o twice (its weights, itself), dS has dP's fp32 sum as well (in e's 2^-18), and the
    outputs are rounded once.  fp16's smallest outputs are off by half of 2^-24, and so are its smallest weights as they are
    held: P times 2^15, which is 2^-40 of a P, and dS times 2^(14 - e) with 2^(e - 1) <= 2.02 |do| |v| < 2^e of the KV head's
    largest rows, which is at most 2^-25 2^(e - 14) <= 2^-38 2.02 |do| |v| of a dS."""
    u = torch.finfo(DT[dtype]).eps / 2
    tiny = 2.0 ** -25 if dtype == "f16" else 0.0
    each_p, each_ds = (2.0 ** -40, 2.0 ** -38 * 2.03) if dtype == "f16" else (0.0, 0.0)
    lse = np.where(np.isfinite(r["lse"]), np.abs(r["lse"]), 0.0)
    bias = 0.0 if slopes is None else float(slopes.max()) * Lk
    e_row = 2.0 ** -20 * r["reach"] + 2.0 ** -22 * (lse + 1.0) + 2.0 ** -22 * bias + (2.0 ** -21 * softcap if softcap else 0.0)
    e = 2.0 * float(e_row.max()) + 2.0 ** -18
    off = u + 2.0 * e                # of P's rounding and of delta's parts
    return {
        "lse": e_row * 2 + 2.0 ** -20,
        "o": u * np.abs(r["o"]) * 1.01 + off * r["o_abs"] + tiny,
        "dv": u * np.abs(r["dv"]) * 1.01 + off * r["dv_abs"] + each_p * r["dv_each"] + tiny,
        "dq": u * np.abs(r["dq"]) * 1.01 + (off + e) * r["dq_abs"] + (2 * off + u) * r["dq_delta"] + each_ds * r["dq_each"] + tiny,
        "dk": u * np.abs(r["dk"]) * 1.01 + (off + e) * r["dk_abs"] + (2 * off + u) * r["dk_delta"] + each_ds * r["dk_each"] + tiny,
    }


def check(got, r, b, what=""):
    """Every element of the named outputs within its bound."""
    for name, t in got.items():
        x, y = t.detach().to("cpu", torch.float64).numpy(), r[name]
        blind = ~np.isfinite(y)
        assert np.array_equal(x[blind], y[blind]), (what, name)
        d = np.abs(np.where(blind, 0.0, x - np.where(blind, 0.0, y)))
        assert np.isfinite(d).all(), (what, name, "not finite")
        share = float((d / np.maximum(np.where(blind, 1.0, b[name]), 1e-300)).max())
        print(f"{what} {name}: largest error {d.max():.3e}, {share:.2f} of its bound", flush=True)
        assert (d <= np.where(blind, 0.0, b[name])).all(), (what, name, share)
