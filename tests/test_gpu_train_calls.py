"""Calls of attention in training that its documents allow beside those of its other tests: scales of either sign and zero under
biases, groups that no power of two divides evenly, many small sequences, one visible key a row."""

import pytest

import paper_2510_08726_amd as pa
from train_cases import bounds, check, draw, oracle64

pytestmark = pytest.mark.gpu


def run(x, **how):
    do, q, k, v, slopes = [None if t is None else t.cuda() for t in x]
    o, lse = pa.attn_fwd_lse(q, k, v, alibi_slopes=slopes, **how)
    return dict(zip(("o", "lse", "dq", "dk", "dv"), (o, lse, *pa.attn_bwd(do, q, k, v, o, lse, alibi_slopes=slopes, **how))))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("scale", [-0.2, 0.0, 1e-6])
def test_scales_under_biases(scale, causal, D):
    for dtype in ("f16", "bf16"):
        x = draw(1, 4, 2, 70, 130, D, dtype, 23, alibi=True)
        how = dict(causal=causal, scale=scale)
        r = oracle64(*x, **how)
        check(run(x, **how), r, bounds(r, dtype, x[4], None, 130), f"{how} {dtype}")


@pytest.mark.parametrize("B,Hq,Hkv,Lq,Lk,D", [(1, 12, 1, 75, 75, 64), (2, 6, 1, 150, 200, 128), (8, 3, 1, 70, 90, 64),
                                              (1, 40, 2, 50, 260, 128), (33, 2, 2, 5, 7, 64), (1, 7, 1, 1, 700, 64)])
def test_groups_and_batches(B, Hq, Hkv, Lq, Lk, D):
    for dtype, how, alibi in (("bf16", dict(causal=True), False), ("f16", dict(causal=True, window=33), True),
                              ("f16", dict(causal=True, softcap=20.0), False), ("bf16", dict(), False)):
        x = draw(B, Hq, Hkv, Lq, Lk, D, dtype, 29, alibi=alibi)
        r = oracle64(*x, **how)
        check(run(x, **how), r, bounds(r, dtype, x[4], how.get("softcap"), Lk), f"{how} {dtype}")
