"""Pins of oracle/serve.py (closed forms and hand-derived values), and the host
function rope_frequencies against it."""

import math

import numpy as np
import pytest
import torch

import paper_2510_08726_amd as pa
from oracle import serve


def test_rope_quarter_turn_and_inverse():
    x = np.arange(8.0).reshape(1, 1, 1, 8)
    f = np.array([math.pi / 2, 0.0])
    half = serve.rope(x, [[1]], f)                    # pairs (0, 2), (1, 3) of the first four dims
    assert np.allclose(half[0, 0, 0], [-2, 1, 0, 3, 4, 5, 6, 7])
    inter = serve.rope(x, [[1]], f, interleaved=True)  # pairs (0, 1), (2, 3)
    assert np.allclose(inter[0, 0, 0], [-1, 0, 2, 3, 4, 5, 6, 7])
    back = serve.rope(half, [[1]], f, transpose=True)
    assert np.allclose(back, x)
    assert np.allclose(serve.rope(x, [[3]], f, magnitude=2.0)[..., :4], 2 * serve.rope(x, [[3]], f)[..., :4])


def test_rope_scores_depend_on_the_distance():
    rng = np.random.default_rng(0)
    q, k = rng.standard_normal((2, 1, 1, 1, 16))
    f = serve.frequencies(16, 10000.0)
    dot = [(serve.rope(q, [[a]], f) * serve.rope(k, [[b]], f)).sum() for a, b in ((5, 2), (105, 102), (3, 0))]
    assert np.allclose(dot, dot[0])


def test_frequencies():
    f = serve.frequencies(64, 10000.0)
    assert f[0] == 1.0 and np.isclose(f[16], 0.01)
    assert np.allclose(serve.frequencies(64, 1e4, "linear", 8.0), f / 8)
    g = serve.frequencies(64, 1e4, "base", 8.0)
    assert g[0] == 1.0 and np.isclose(g[-1], f[-1] / 8)
    h = serve.frequencies(64, 1e4, "parts", 8.0, 4096, 1.0, 32.0)
    assert h[0] == f[0] and np.isclose(h[-1], f[-1] / 8) and (np.diff(h) < 0).all()


@pytest.mark.parametrize("kw", [dict(), dict(scaling="linear", factor=4.0), dict(scaling="base", factor=4.0),
                                dict(scaling="parts", factor=8.0, original_length=8192, slow=1.0, fast=4.0)], ids=str)
@pytest.mark.parametrize("R,base", [(4, 100.0), (64, 1e4), (128, 5e5)])
def test_library_frequencies(R, base, kw):
    got = pa.rope_frequencies(R, base, **kw)
    assert got.dtype == torch.float64
    assert np.allclose(got.numpy(), serve.frequencies(R, base, **kw), rtol=1e-14)


def test_held_by_hand():
    x = np.zeros(32)
    x[:12] = [7.0, 6.5, 5.0, 5.1, 3.5, 2.5, 1.75, 1.25, 0.75, 0.25, 0.26, -0.5]
    code, scale, value = serve.held(x, "f16")
    assert scale == [127]                              # 7 <= 7 * 2^0
    assert list(value[:12]) == [6, 6, 4, 6, 4, 2, 2, 1, 1, 0, 0.5, -0.5]
    assert list(code[:12]) == [7, 7, 6, 7, 6, 4, 4, 2, 2, 0, 1, 9]
    x[0] = 7.01
    code, scale, value = serve.held(x, "f16")
    assert scale == [128] and value[0] == 8.0          # 3.505 * 2 -> 4 * 2
    assert serve.held(np.full(32, 1e6), "f16")[2][0] == 6 * 2.0 ** 13
    assert serve.held(np.full(32, 2.0 ** -14), "f16")[2][0] == 2.0 ** -14
    assert serve.held(np.full(32, 2.0 ** -15.1), "f16")[2][0] == 0.0
    assert np.isnan(serve.held(np.r_[np.inf, np.zeros(31)], "bf16")[2]).all()
    assert serve.held(np.r_[np.inf, np.zeros(31)], "bf16")[1] == [255]


def test_held_is_no_further_than_a_fifth():
    """An element is off by half a step of its binade at most, the largest by a seventh
    (7 held as 6): a sixth of the block's largest value in all."""
    rng = np.random.default_rng(1)
    x = rng.standard_normal((200, 64)) * np.exp2(rng.integers(-5, 6, (200, 1)))
    _, _, v = serve.held(x, "bf16")
    top = np.abs(x.reshape(200, 2, 32)).max(-1).repeat(32, -1)
    assert (np.abs(v - x) <= top / 4 + 1e-12).all()
    assert np.sqrt(((v - x) ** 2).mean() / (x ** 2).mean()) < 0.13


def test_pack_unpack():
    rng = np.random.default_rng(2)
    page, D = 16, 64
    cache = rng.integers(0, 256, (3, 2, serve.page_bytes(page, D))).astype(np.uint8)
    assert serve.page_bytes(page, D) == pa.kv4_page_bytes(page, D) == 1088
    k, v = rng.standard_normal((2, D))
    ck, sk, vk = serve.held(k, "bf16")
    cv, sv, vv = serve.held(v, "bf16")
    was = cache.copy()
    serve.pack(cache, 21, 1, ck, sk, cv, sv, page, D)
    a, b = serve.unpack(cache, 21, 1, page, D)
    assert np.array_equal(a, vk) and np.array_equal(b, vv)
    assert (cache != was).sum() <= 2 * (D // 2 + D // 32)
    assert np.array_equal(cache[[0, 2]], was[[0, 2]]) and np.array_equal(cache[1, 0], was[1, 0])


def test_slots_by_hand():
    table = np.array([[9, -1, -1], [4, 5, -1], [7, -1, -1]])
    out, pos, new, taken, t = serve.slots([3, 8, 0], [3, 2, 1], table, [20, 21, 22], 4, 3)
    assert out.tolist() == [[39, 80, 81], [84, 85, -1], [88, -1, -1]]
    assert pos.tolist() == [[3, 4, 5], [8, 9, 10], [0, 1, 2]]
    assert new.tolist() == [6, 10, 1] and taken == 3
    assert t.tolist() == [[9, 20, -1], [4, 5, 21], [22, -1, -1]]
    out, _, new, taken, _ = serve.slots([3, 8, 0], [3, 2, 1], table, [20], 4, 3)      # pages run out
    assert out.tolist() == [[39, 80, 81], [-1, -1, -1], [-1, -1, -1]] and new.tolist() == [6, 8, 0] and taken == 1


def test_decode_is_the_attention_of_each_request():
    rng = np.random.default_rng(3)
    q = rng.standard_normal((2, 4, 1, 16))
    k, v = rng.standard_normal((2, 2, 5, 16))
    o, mean = serve.decode(q, [k, k[:, :0]], [v, v[:, :0]], scale=0.25)
    for h in range(4):
        s = 0.25 * k[h // 2] @ q[0, h, 0]
        w = np.exp(s - s.max())
        assert np.allclose(o[0, h, 0], w @ v[h // 2] / w.sum()) and np.allclose(mean[0, h, 0], w @ abs(v[h // 2]) / w.sum())
    assert not o[1].any()
