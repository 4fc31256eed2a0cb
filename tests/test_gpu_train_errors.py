"""The errors of attention's outputs in training, as root mean squares against 64 bits: those of the roundings that the kernels choose
(train_errors.py)."""

import math

import numpy as np
import pytest
import torch

import paper_2510_08726_amd as pa
import train_errors as te

pytestmark = pytest.mark.gpu


def run(case, x):
    do, q, k, v, slopes = [None if t is None else t.cuda() for t in x]
    how = dict(causal=case[6], alibi_slopes=slopes, softcap=case[8], window=case[9])
    o, lse = pa.attn_fwd_lse(q, k, v, **how)
    got = dict(zip(("o", "lse", "dq", "dk", "dv"), (o, lse, *pa.attn_bwd(do, q, k, v, o, lse, **how))))
    return {n: t.cpu().double().numpy() for n, t in got.items()}


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("case", te.CASES)
def test_errors_are_those_of_the_roundings(case, dtype):
    x = te.inputs(case, dtype)
    want, emulated = te.both64(case, x, dtype)
    got = run(case, x)
    share = te.shares({n: t for n, t in got.items() if n != "lse"}, want, emulated)
    print(case, dtype, share, flush=True)
    # lse: one rounding of itself, and the errors of the scores that it sums (2^-20 of their sums of magnitudes) and of its
    # logarithm.
    seen = np.isfinite(want["lse"])
    assert np.array_equal(np.isfinite(got["lse"]), seen)
    off = np.abs(np.where(seen, got["lse"] - np.where(seen, want["lse"], 0.0), 0.0))
    most = 2.0 ** -24 * 1.01 * np.abs(np.where(seen, want["lse"], 0.0)) + 2.0 ** -19 * (want["reach"] + 1.0)
    if case[8]:
        most = most + 2.0 ** -21 * case[8]
    assert (off <= most).all(), float((off / most).max())
    assert all(s <= te.MORE for s in share.values()), share
    assert not any(math.isnan(s) for s in share.values())
