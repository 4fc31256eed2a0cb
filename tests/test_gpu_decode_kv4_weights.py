"""The softmax weights of the 4-bit decode: what 16-bit operands of the matrix unit must not cost."""

import numpy as np
import pytest
import torch

import paper_2510_08726_amd as pa
from oracle import serve
from paper_2510_08726_amd.workloads import alibi_slopes, random_tensors
from gpu_common import host64

pytestmark = pytest.mark.gpu

DT = {"f16": torch.float16, "bf16": torch.bfloat16}


def _i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def _requests(lens, Hkv, D, dtype, page, seed):
    """A cache whose pages lie in order, and the values of each request as held."""
    M = max(-(-n // page) for n in lens)
    table = np.arange(len(lens) * M).reshape(len(lens), M)
    cache = torch.zeros(table.size, Hkv, pa.kv4_page_bytes(page, D), dtype=torch.uint8, device="cuda")
    held = [[], []]
    for b, n in enumerate(lens):
        k, v = random_tensors([(1, Hkv, n, D)] * 2, dtype, seed + 10 * b)
        slots = table[b, np.arange(n) // page] * page + np.arange(n) % page
        pa.kv4_append(k.cuda(), v.cuda(), cache, torch.tensor(slots[None], device="cuda"))
        for h, x in zip(held, (k, v)):
            h.append(serve.held(host64(x[0]), dtype)[2])
    return cache, _i32(table), held


@pytest.mark.parametrize("Hq,Hkv,alibi,softcap", [(8, 2, False, None), (2, 2, True, None), (20, 1, False, 2.0),
                                                  (40, 1, True, 2.0)])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_weights_keep_twice_the_bits_of_the_type(dtype, D, Hq, Hkv, alibi, softcap):
    """A weight is the sum of two values of the type: the second holds what the first leaves (half
    a step of the weight at most) to half a step of its own, so half ** 2 of the weight is lost.
    Scores and exponentials in 32 bits are off by under 2e-5 of a weight for scores up to 60; what
    fp16 cannot hold of a weight is 2^-25 at most, where the largest is 1 or more.  The output is rounded once."""
    lens = [2, 3, 5, 17, 40, 333, 2000]
    cache, table, (ks, vs) = _requests(lens, Hkv, D, dtype, 32, Hq)
    q, = random_tensors([(len(lens), Hq, 1, D)], dtype, 5)
    sl = alibi_slopes(Hq) if alibi else None
    o = pa.attn_decode_kv4(q.cuda(), cache, table, _i32(lens), softcap=softcap,
                           alibi_slopes=None if sl is None else sl.cuda())
    ref, mean = serve.decode(host64(q), ks, vs, scale=D ** -0.5, slopes=None if sl is None else host64(sl),
                             softcap=softcap)
    half = torch.finfo(q.dtype).eps / 2
    most = max(np.abs(v).max() for v in vs)
    tiny = 2.0 ** -25 * (1 + most * np.array(lens)[:, None, None, None]) if dtype == "f16" else 0.0   # and the output's
    tol = half * np.abs(ref) + 1.01 * (half ** 2 + 2e-5) * mean + tiny + 1e-6
    err = np.abs(host64(o) - ref)
    print(f"{dtype} {D} {Hq}: worst {np.max(err / tol):.3f} of the tolerance", flush=True)
    assert (err <= tol).all()
