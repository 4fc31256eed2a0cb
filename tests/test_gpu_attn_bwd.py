"""Attention in training on the GPU: attn_fwd_lse and attn_bwd against the gradients in 64 bits."""

import pytest
import torch

import paper_2510_08726_amd as pa
from train_cases import bounds, check, draw, oracle64

pytestmark = pytest.mark.gpu

# (B, Hq, Hkv, Lq, Lk, D, causal, alibi, softcap, window)
CASES = [
    (1, 1, 1, 1, 1, 64, False, False, None, None),          # one token
    (2, 3, 3, 1, 37, 64, True, False, None, None),          # one query row
    (1, 2, 2, 32, 32, 64, False, False, None, None),        # one whole tile
    (1, 2, 1, 33, 31, 128, False, False, None, None),       # a tile and a row, a ragged tile
    (2, 4, 2, 130, 257, 64, False, False, None, None),
    (1, 4, 4, 128, 128, 128, True, False, None, None),
    (2, 8, 2, 200, 200, 128, True, False, None, None),      # grouped heads
    (1, 5, 1, 161, 161, 64, True, False, None, None),       # a group of five
    (1, 6, 3, 97, 300, 64, True, False, None, None),        # more keys than queries
    (1, 4, 2, 300, 97, 128, True, False, None, None),       # rows that see no key
    (1, 2, 2, 65, 1, 64, True, False, None, None),          # all rows but one see no key
    (1, 4, 4, 150, 150, 64, False, True, None, None),       # biases
    (2, 4, 2, 300, 333, 128, True, True, None, None),
    (1, 2, 1, 190, 190, 64, True, False, 5.0, None),        # capped scores
    (1, 4, 2, 129, 260, 128, True, False, 50.0, None),
    (1, 2, 2, 300, 300, 64, True, False, None, 1),          # windows
    (1, 4, 2, 300, 420, 128, True, False, None, 77),
    (1, 2, 1, 420, 300, 64, True, False, 20.0, 40),
    (1, 4, 4, 333, 333, 128, True, True, None, 100),
    (1, 2, 2, 100, 500, 64, True, False, None, 30),         # keys that no row sees
    (1, 16, 1, 40, 70, 128, True, False, None, None),       # sixteen heads share
    (1, 2, 1, 1100, 1100, 128, True, False, None, None),    # long
    (1, 1, 1, 50, 33100, 64, True, False, None, None),      # over 256 blocks of keys
    (1, 2, 2, 33100, 50, 128, False, False, None, None),    # over 256 blocks of rows
]


def run(do, q, k, v, slopes, strided=False, **how):
    x = [t.cuda() for t in (do, q, k, v)]
    if strided:
        x[0] = x[0].transpose(1, 2).contiguous().transpose(1, 2)
    how["alibi_slopes"] = None if slopes is None else slopes.cuda()
    o, lse = pa.attn_fwd_lse(*x[1:], **how)
    dq, dk, dv = pa.attn_bwd(*x, o, lse, **how)
    torch.cuda.synchronize()
    return {"o": o, "lse": lse, "dq": dq, "dk": dk, "dv": dv}


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("case", CASES)
def test_gradients(case, dtype):
    B, Hq, Hkv, Lq, Lk, D, causal, alibi, softcap, window = case
    x = draw(B, Hq, Hkv, Lq, Lk, D, dtype, seed=sum(case[:6]), alibi=alibi)
    how = {"causal": causal, "softcap": softcap, "window": window}
    r = oracle64(*x, **how)
    got = run(*x, strided=Lq % 2 == 0, **how)
    check(got, r, bounds(r, dtype, x[4], softcap, Lk), f"{case} {dtype}")
