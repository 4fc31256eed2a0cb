"""The 64-bit definitions behind the tests of the training operators, pinned apart from the GPU."""

import numpy as np
import pytest
import torch

from oracle import train
from train_cases import draw, oracle64


@pytest.mark.parametrize("causal,alibi,softcap,window,Lq,Lk", [
    (False, False, None, None, 9, 11), (True, False, None, None, 20, 33), (True, False, None, None, 33, 20),
    (True, True, None, 7, 33, 20), (True, False, 3.0, 9, 20, 30), (False, True, None, None, 9, 11)])
def test_attention_gradients_are_autograds(causal, alibi, softcap, window, Lq, Lk):
    do, q, k, v, slopes = draw(2, 4, 2, Lq, Lk, 64, "f16", 3, alibi=alibi)
    r = oracle64(do, q, k, v, slopes, causal=causal, softcap=softcap, window=window)
    Q, K, V = [t.double().requires_grad_() for t in (q, k, v)]
    s = (Q.reshape(2, 2, 2, Lq, 64) @ K[:, :, None].transpose(-1, -2)) / 8
    if softcap:
        s = softcap * torch.tanh(s / softcap)
    ahead = torch.arange(Lq)[:, None] + Lk - Lq - torch.arange(Lk)[None]
    if alibi:
        s = s - slopes.double().reshape(2, 2, 1, 1) * ahead
    seen = ahead >= 0 if causal else torch.ones(Lq, Lk, dtype=torch.bool)
    if window:
        seen = seen & (ahead < window)
    some = seen.any(-1)
    s = s.masked_fill(~seen, -1e300)
    o = (torch.softmax(s, -1) * some[:, None] @ V[:, :, None]).reshape(2, 4, Lq, 64)
    o.backward(do.double())
    for name, t in (("o", o), ("dq", Q.grad), ("dk", K.grad), ("dv", V.grad)):
        assert np.abs(r[name] - t.detach().numpy()).max() <= 1e-12, name
    lse = torch.logsumexp(s, -1).reshape(2, 4, Lq).masked_fill(~some, -np.inf).detach().numpy()
    assert np.array_equal(np.isfinite(r["lse"]), np.isfinite(lse))
    assert np.abs(np.where(np.isfinite(lse), r["lse"] - np.where(np.isfinite(lse), lse, 0), 0)).max() <= 1e-12


def test_attention_gradients_are_difference_quotients():
    do, q, k, v, _ = draw(1, 2, 1, 7, 9, 64, "f16", 5)
    how = dict(causal=True, softcap=20.0)
    r = oracle64(do, q, k, v, None, **how)
    x = {"q": q.double().numpy(), "k": k.double().numpy(), "v": v.double().numpy()}
    rng = np.random.default_rng(1)
    for name, t in x.items():
        step = rng.standard_normal(t.shape)
        f = []
        for sign in (1, -1):
            y = {**x, name: t + sign * 1e-5 * step}
            o = train.attention_grad(do.double().numpy(), y["q"], y["k"], y["v"], scale=0.125, **how)["o"]
            f.append((o * do.double().numpy()).sum())
        assert abs((f[0] - f[1]) / 2e-5 - (r["d" + name] * step).sum()) <= 1e-7 * np.abs(r["d" + name] * step).sum()


@pytest.mark.parametrize("weight,above,offset", [(True, True, 0.0), (True, False, 1.0), (False, True, 3.0)])
def test_norm_gradients_are_autograds(weight, above, offset):
    g = torch.Generator().manual_seed(1)
    h = torch.randn((5, 33), generator=g, dtype=torch.float64).requires_grad_()
    w = torch.randn(33, generator=g, dtype=torch.float64).requires_grad_()
    dy, dh = torch.randn((5, 33), generator=g, dtype=torch.float64), torch.randn((5, 33), generator=g, dtype=torch.float64)
    rstd = (h.square().mean(-1) + 1e-3).rsqrt()
    y = h * rstd[:, None] * (w + offset if weight else 1.0)
    loss = (y * dy).sum() + ((h * dh).sum() if above else 0.0)
    loss.backward()
    wn = w.detach().numpy() if weight else None
    want, r = train.rmsnorm(h.detach().numpy(), wn, 1e-3, offset)
    assert np.abs(want - y.detach().numpy()).max() <= 1e-13 and np.abs(r - rstd.detach().numpy()).max() <= 1e-13
    dx, dw, *_ = train.rmsnorm_grad(dy.numpy(), h.detach().numpy(), r, wn, dh.numpy() if above else None, offset)
    assert np.abs(dx - h.grad.numpy()).max() <= 1e-12
    if weight:
        assert np.abs(dw - w.grad.numpy()).max() <= 1e-12


def test_codes_are_the_nearest():
    """Against PyTorch's own rounding to the 8-bit types, at the middles between codes as well."""
    grid = torch.arange(-126, 127, dtype=torch.int8).view(torch.uint8)
    e4m3 = torch.arange(0, 127, dtype=torch.uint8).view(torch.float8_e4m3fn).double()
    z = torch.cat([e4m3, (e4m3[1:] + e4m3[:-1]) / 2, torch.linspace(0, 448, 5001, dtype=torch.float64)])
    z = torch.cat([z, -z, torch.tensor([448.0])])[None]                 # the largest is 448: a scale of 1
    values, s = train.codes8(z.numpy(), "e4m3", 0)
    assert s.tolist() == [[1.0]]
    # (exact in fp32: the steps of linspace are rounded there first, and compared as such)
    z32 = z.float()
    values32, _ = train.codes8(z32.double().numpy(), "e4m3", 0)
    assert np.array_equal(values32, z32.to(torch.float8_e4m3fn).double().numpy())
    z = torch.cat([torch.arange(-254, 255, dtype=torch.float64) / 2, torch.tensor([127.0], dtype=torch.float64)])[None]
    values, s = train.codes8(z.numpy(), "int8", 0)
    assert s.tolist() == [[1.0]] and np.array_equal(values, z.round().numpy())
    assert len(grid) == 253


def test_codes_of_groups():
    y = np.zeros((2, 70))
    y[0, :32] = np.linspace(-3, 3, 32)
    y[0, 40] = np.inf
    y[1, 69] = -5.0
    values, s = train.codes8(y, "int8", 32)
    assert s.shape == (2, 3) and np.isnan(s[0, 1]) and (values[0, 32:64] == 0).all()
    assert s[0, 0] == np.float32(3 / 127) and abs(values[0, 0]) == 127 and s[0, 2] == 0
    assert s[1, 2] == np.float32(5 / 127) and values[1, 69] == -127 and (values[1, :64] == 0).all()
