"""SoftCap of the 4-bit decode with caps from far under the scores to far above them."""

import numpy as np
import pytest
import torch

import paper_2510_08726_amd as pa
from oracle import serve
from paper_2510_08726_amd.workloads import alibi_slopes, random_tensors
from gpu_common import host64

pytestmark = pytest.mark.gpu


def _i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("cap", [1e-44, 1e-30, 0.5, 30.0, 64.0, 65.0, 100.0, 1e3, 1e5, 1e30, 3.4e38])
@pytest.mark.parametrize("Hq,Hkv,D,alibi", [(8, 2, 128, False), (8, 2, 64, True), (20, 1, 64, False), (20, 1, 128, True)])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_any_cap(dtype, Hq, Hkv, D, alibi, cap):
    """Scores up to 60.  In 32 bits the score is off by 4 roundings (60 * 4 * 2^-24 = 1.4e-5), and
    the capped one by 2^-22 of the cap where that is 64 or less (1.6e-5), else by under 3e-7 of
    itself (1.8e-5); the exponential and the sums by under 1e-5: so 5e-5 of a weight, and for both
    heads' and sums' weights twice that of the weighted mean of |v|.  A weight's two values of the
    type lose half a step squared, and what fp16 cannot hold of it is 2^-25; the output is rounded once."""
    lens, page = [1, 70, 600], 32
    M = -(-max(lens) // page)
    table = np.arange(len(lens) * M).reshape(len(lens), M)
    cache = torch.zeros(table.size, Hkv, pa.kv4_page_bytes(page, D), dtype=torch.uint8, device="cuda")
    ks, vs = [], []
    for b, n in enumerate(lens):
        k, v = random_tensors([(1, Hkv, n, D)] * 2, dtype, 10 * b)
        slots = table[b, np.arange(n) // page] * page + np.arange(n) % page
        pa.kv4_append(k.cuda(), v.cuda(), cache, torch.tensor(slots[None], device="cuda"))
        ks.append(serve.held(host64(k[0]), dtype)[2])
        vs.append(serve.held(host64(v[0]), dtype)[2])
    q, = random_tensors([(len(lens), Hq, 1, D)], dtype, 5)
    most = max(np.abs(np.einsum("hd,gnd->hgn", host64(q)[b, :, 0], k)).max() for b, k in enumerate(ks))
    scale = float(np.float32(60.0 / most))
    sl = alibi_slopes(Hq) if alibi else None
    o = pa.attn_decode_kv4(q.cuda(), cache, _i32(table), _i32(lens), scale=scale, softcap=cap,
                           alibi_slopes=None if sl is None else sl.cuda())
    ref, mean = serve.decode(host64(q), ks, vs, scale=scale, slopes=None if sl is None else host64(sl),
                             softcap=float(np.float32(cap)))
    half = torch.finfo(q.dtype).eps / 2
    tiny = 2.0 ** -25 * (1 + 6 * np.array(lens)[:, None, None, None]) if dtype == "f16" else 0.0
    tol = half * np.abs(ref) + (1.01 * half ** 2 + 1e-4) * mean + tiny + 1e-6
    err = np.abs(host64(o) - ref)
    print(f"{dtype} {D} {Hq} cap {cap}: worst {np.max(err / tol):.3f} of the tolerance", flush=True)
    assert (err <= tol).all()


@pytest.mark.parametrize("cap", [1e-44, 1e-30, 1.0, 1e5, 3.4e38])
def test_scores_of_zero(cap):
    """No score, no cap: the mean of V (whole numbers here, of 32 tokens: exact)."""
    D, n = 64, 32
    v = torch.tensor(np.tile([1.0, 2.0, 3.0, 6.0], n * D // 4).reshape(1, 1, n, D), dtype=torch.float16, device="cuda")
    cache = torch.zeros(1, 1, pa.kv4_page_bytes(32, D), dtype=torch.uint8, device="cuda")
    pa.kv4_append(torch.ones_like(v), v, cache, torch.arange(n, device="cuda")[None])
    q = torch.zeros(1, 1, 1, D, dtype=torch.float16, device="cuda")
    o = pa.attn_decode_kv4(q, cache, _i32([[0]]), _i32([n]), softcap=cap)
    assert torch.equal(o[0, 0, 0], v[0, 0, 0])


@pytest.mark.parametrize("cap", [30.0, 1e5, 3.4e38])
def test_infinite_scores_reach_the_cap(cap):
    """Half of the scores are inf, half -inf: capped, the first weigh the same and the others nothing
    (e^-2 cap of a weight)."""
    D, n = 64, 32
    k, v = torch.zeros(2, 1, 1, n, D, dtype=torch.float16, device="cuda")
    k[..., 0::2, 0], k[..., 1::2, 0] = 1.0, -1.0
    v[..., 0::2, :], v[..., 1::2, :] = 2.0, 6.0
    cache = torch.zeros(1, 1, pa.kv4_page_bytes(32, D), dtype=torch.uint8, device="cuda")
    pa.kv4_append(k, v, cache, torch.arange(n, device="cuda")[None])
    q = torch.zeros(1, 1, 1, D, dtype=torch.float16, device="cuda")
    q[..., 0] = float("inf")
    o = pa.attn_decode_kv4(q, cache, _i32([[0]]), _i32([n]), softcap=cap)
    assert (o == 2.0).all()
