"""The norm with the residual's addition on the GPU: rmsnorm_add, its gradients and its 8-bit form, against 64 bits."""

import numpy as np
import pytest
import torch

import paper_2510_08726_amd as pa
from oracle import train

pytestmark = pytest.mark.gpu

DT = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
TINY = {"f16": 2.0 ** -25, "bf16": 2.0 ** -134, "f32": 2.0 ** -150}      # half of the smallest values' distance
U = {k: torch.finfo(v).eps / 2 for k, v in DT.items()}
TYPES = [("f16", "f16"), ("f16", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")]
# Rows and their lengths: one element, odd ones, each number of lanes and steps, more rows than workgroups.
SIZES = [(1, 1), (3, 5), (1, 64), (7, 512), (5, 513), (2, 1000), (33, 1024), (9, 4096), (4, 8191), (3, 8200), (2, 16384),
         (1, 20001), (2, 32768), (300, 97), (2100, 640)]


def draw(N, M, dtype, wide, seed):
    g = torch.Generator().manual_seed(seed)
    t = lambda *s: torch.randn(s, generator=g)     # noqa: E731
    size = 1.0 + 7.0 * (torch.arange(M) % 97 == 31)
    return (t(N, M).to(DT[dtype]), (3 * t(N, M) * size).to(DT[wide]), (1 + 0.2 * t(M)).to(DT[dtype]),
            t(N, M).to(DT[dtype]), t(N, M).to(DT[wide]))


def np64(t):
    return t.detach().to("cpu", torch.float64).numpy()


def cuda(*ts):
    return [None if t is None else t.cuda() for t in ts]


@pytest.mark.parametrize("N,M", SIZES)
@pytest.mark.parametrize("types", TYPES)
def test_norm(N, M, types):
    dtype, wide = types
    x, res, w, _, _ = draw(N, M, dtype, wide, N + M)
    for residual, weight, offset, eps in ((res, w, 0.0, 1e-6), (None, w, 1.0, 1e-2), (res, None, 3.0, 0.0)):
        gx, gr, gw = cuda(x, residual, weight)
        y, h, rstd = pa.rmsnorm_add(gx, gr, gw, eps=eps, weight_offset=offset)
        torch.cuda.synchronize()
        if residual is None:
            assert h is gx
        else:
            assert torch.equal(h.cpu(), (x.float() + res.float()).to(DT[wide]))
        want, r = train.rmsnorm(np64(h), None if weight is None else np64(weight), eps, offset)
        assert np.all(np.abs(np64(rstd) - r) <= 2.0 ** -24 * 1.01 * r)
        # rstd, weight + offset and two products in fp32, the output's rounding
        assert y.dtype == x.dtype
        assert np.all(np.abs(np64(y) - want) <= (U[dtype] * 1.01 + 4.05 * 2.0 ** -24) * np.abs(want) + TINY[dtype])


@pytest.mark.parametrize("N,M", SIZES)
@pytest.mark.parametrize("types", TYPES)
def test_norm_gradients(N, M, types):
    dtype, wide = types
    _, h, w, dy, dh = draw(N, M, dtype, wide, N + M + 1)
    rstd = (h.double().square().mean(-1) + 1e-6).rsqrt().float()
    for weight, above, offset in ((w, dh, 0.0), (w, None, 1.0), (None, dh, 0.0)):
        ghs = cuda(dy, h, rstd, weight, above)
        dx, dres, dw = pa.rmsnorm_add_bwd(*ghs, weight_offset=offset)
        torch.cuda.synchronize()
        assert dx.dtype == dy.dtype and dres.dtype == h.dtype and (dres is dx) == (dtype == wide)
        d, want_w, terms, mean, size_w = train.rmsnorm_grad(np64(dy), np64(h), np64(rstd), None if weight is None else np64(weight),
                                                            None if above is None else np64(above), offset)
        # A lane adds up to 32 products one after another, ten joins follow; eight roundings of the terms.
        off = 2.0 ** -24 * (8 * terms + 50 * mean)
        for t, name in ((dx, dtype), (dres, wide)):
            assert np.all(np.abs(np64(t) - d) <= U[name] * 1.01 * np.abs(d) + off + TINY[name]), (name, weight is None)
        if weight is None:
            assert dw is None
        else:
            # The rows of a partial, an eighth of the (at most 1024, in fours) partials, and eight sums.
            chain = -(-N // 1024) + 4096 // 8 + 8 + 3 if N > 1024 else N // 8 + 15
            assert dw.dtype == torch.float32
            assert np.all(np.abs(np64(dw) - want_w) <= 2.0 ** -24 * chain * size_w + 2.0 ** -150)


@pytest.mark.parametrize("N,M", SIZES)
@pytest.mark.parametrize("code", ["e4m3", "int8"])
@pytest.mark.parametrize("types", TYPES)
def test_norm_in_8_bits(N, M, code, types):
    dtype, wide = types
    x, res, w, _, _ = draw(N, M, dtype, wide, N + M + 2)
    q_type = torch.int8 if code == "int8" else torch.float8_e4m3fn
    for residual, weight, offset, group in ((res, w, 0.0, 0), (None, w, 1.0, 128), (res, None, 0.0, 32), (res, w, 1.0, 256),
                                            (res, w, 0.0, 64)):
        gx, gr, gw = cuda(x, residual, weight)
        rstd = torch.empty(N, device="cuda")
        q, scales, h = pa.rmsnorm_add_quant(gx, gr, gw, dtype=q_type, group=group, weight_offset=offset, rstd=rstd)
        torch.cuda.synchronize()
        if residual is not None:
            assert torch.equal(h.cpu(), (x.float() + res.float()).to(DT[wide]))
        want, r = train.rmsnorm(np64(h), None if weight is None else np64(weight), 1e-6, offset)
        assert np.all(np.abs(np64(rstd) - r) <= 2.0 ** -24 * 1.01 * r)
        values, s = train.codes8(want, code, group)
        assert q.dtype == q_type and scales.shape == s.shape
        assert np.array_equal(scales.cpu().numpy(), s)
        assert np.array_equal(np64(q.float()), values)
        for t in ("f16", "bf16", "f32"):
            y = pa.quant8_load(q, scales, group=group, dtype=DT[t])
            back = (q.cpu().float() * torch.from_numpy(np.repeat(s, group or M, 1)[:, :M])).to(DT[t])
            assert torch.equal(y.cpu(), back)
