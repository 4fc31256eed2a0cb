"""The errors of attention's outputs in training, as root mean squares against 64 bits: those of the roundings that the kernels choose
(train_errors.py), where a log-sum-exp in the thousands stands beside the scores too."""

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
@pytest.mark.parametrize("case", te.CASES + te.FAR)
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


def test_a_zero_slope_and_slopes_of_both_signs():
    """Heads of one call, each with its own origin; a slope of 0 is no bias."""
    B, H, L, D = 1, 4, 500, 64
    g = torch.Generator().manual_seed(3)
    do, q, k, v = [torch.randn((B, H, L, D), generator=g).to(torch.float16).cuda() for _ in range(4)]
    for causal in (False, True):
        slopes = torch.tensor([0.5, 0.0, -0.0, -0.5], device="cuda")
        o, lse = pa.attn_fwd_lse(q, k, v, causal=causal, alibi_slopes=slopes)
        grads = pa.attn_bwd(do, q, k, v, o, lse, causal=causal, alibi_slopes=slopes)
        for h in range(H):
            one = [t[:, h:h + 1].contiguous() for t in (do, q, k, v)]
            how = dict(causal=causal, alibi_slopes=slopes[h:h + 1].clone())
            o1, lse1 = pa.attn_fwd_lse(*one[1:], **how)
            alone = (o1, lse1, *pa.attn_bwd(*one, o1, lse1, **how))
            for a, b in zip((o, lse, *grads), alone):
                # (Another division of the blocks sums in another order, and fp16's power of two may differ.)
                d = (a[:, h:h + 1].float() - b.float()).abs().max()
                assert d <= 2.0 ** -9 * b.float().abs().max(), (causal, h)
