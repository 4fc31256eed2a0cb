"""Rotary positions on the GPU against the definition in 64 bits: both pairings,
parts of the head, vectors and single elements, strided inputs, far positions,
the gradient, streams and graphs."""

import numpy as np
import pytest
import torch

import paper_2510_08726_amd as pa
from oracle import serve
from paper_2510_08726_amd.workloads import random_tensors
from gpu_common import host64

pytestmark = pytest.mark.gpu

DT = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def _tolerance(x, y, dtype, positions, freqs, R, interleaved, magnitude):
    """Half a step of the type, and of the 32-bit arithmetic: the reduced angle (two
    roundings of at most pi / 4: 1.5e-7), the series (1.2e-7), the magnitude, the two products
    and their sum (2^-24 each), 6e-7 of |a| + |b| in all; the angle's 64-bit product and
    its reduction are off by 3 roundings of 2^-53 of it."""
    a = np.abs(x)
    n = R // 2
    pair = np.zeros_like(a)
    if interleaved:
        pair[..., 0:R:2] = pair[..., 1:R:2] = a[..., 0:R:2] + a[..., 1:R:2]
    else:
        pair[..., :n] = pair[..., n:R] = a[..., :n] + a[..., n:R]
    far = 3 * 2.0 ** -53 * np.abs(np.asarray(positions, dtype=np.float64)).max() * np.max(freqs)
    return torch.finfo(dtype).eps / 2 * np.abs(y) + abs(magnitude) * pair * (6e-7 + far)


def _check(got, x, positions, freqs, interleaved, magnitude, bwd, what):
    ref = serve.rope(host64(x), positions, freqs, interleaved=interleaved, magnitude=magnitude, transpose=bwd)
    tol = _tolerance(host64(x), ref, x.dtype, positions, freqs, 2 * len(freqs), interleaved, magnitude)
    err = np.abs(host64(got) - ref)
    # fp16 values under 2^-14 are spaced 2^-24, and are off by half of that.
    tol = tol + (2.0 ** -25 if x.dtype == torch.float16 else 0.0)
    print(f"{what}: worst {np.max(err / (tol + 1e-300)):.3f} of the tolerance", flush=True)
    assert (err <= tol).all(), what
    R = 2 * len(freqs)
    assert torch.equal(got[..., R:], x[..., R:])


def _views(B, H, L, D, dtype, seed, layout):
    if layout == "plain":
        return random_tensors([(B, H, L, D)], dtype, seed, device="cuda")[0]
    if layout == "projection":     # queries, keys and values side by side
        x, = random_tensors([(B, L, 2 * H + 1, D)], dtype, seed, device="cuda")
        return x[:, :, 1:H + 1].transpose(1, 2)
    x, = random_tensors([(B, H, L, D + 1)], dtype, seed, device="cuda")       # rows at odd elements
    return x[..., 1:]


@pytest.mark.parametrize("layout", ["plain", "projection", "odd"])
@pytest.mark.parametrize("D,R", [(128, 128), (64, 32), (64, 24), (128, 8), (20, 12), (6, 2), (2, 2)])
@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True], ids=["half", "interleaved"])
def test_rope(dtype, interleaved, D, R, layout):
    freqs = serve.frequencies(R, 10000.0)
    for n, (B, L, Hq, Hkv) in enumerate([(1, 1, 1, 1), (3, 7, 5, 2), (2, 129, 3, 3)]):
        q, k = (_views(B, H, L, D, DT[dtype], 10 * n + i, layout) for i, H in enumerate((Hq, Hkv)))
        pos = np.random.default_rng(n).integers(-50, 5000, (B, L))
        f = torch.tensor(freqs, device="cuda")
        for bwd, fn in ((False, pa.rope_fwd), (True, pa.rope_bwd)):
            qo, ko = fn(q, k, torch.tensor(pos, dtype=torch.int32, device="cuda"), f, interleaved=interleaved,
                        magnitude=1.1)
            for t, o in ((q, qo), (k, ko)):
                assert o.is_contiguous() and o.dtype == t.dtype
                _check(o, t, pos, freqs, interleaved, np.float32(1.1), bwd, (dtype, D, R, layout, B, L, bwd))


@pytest.mark.parametrize("D,R", [(128, 128), (128, 64), (64, 24), (40, 20)])
@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True], ids=["half", "interleaved"])
def test_many_tokens_are_turned_like_few(dtype, interleaved, D, R):
    """Enough rows that a thread takes several heads (a number that its four do not divide,
    keys behind queries): the same bits as call by call on a few tokens."""
    L, f = 4300, pa.rope_frequencies(R, device="cuda")      # 68 MB of 16-bit outputs at D = 128: streamed
    q, k = (_views(2, H, L, D, DT[dtype], 40 + H, "projection") for H in (25, 6))
    pos = torch.randint(0, 100000, (2, L), dtype=torch.int32, device="cuda")
    whole = pa.rope_fwd(q, k, pos, f, interleaved=interleaved)
    for lo in range(0, L, 410):
        some = pa.rope_fwd(q[:, :, lo:lo + 410], k[:, :, lo:lo + 410], pos[:, lo:lo + 410].contiguous(), f,
                           interleaved=interleaved)
        one = pa.rope_fwd(q[:, :1, lo:lo + 3], None, pos[:, lo:lo + 3].contiguous(), f, interleaved=interleaved)[0]
        for a, b in zip(whole, some):
            assert torch.equal(a[:, :, lo:lo + 410], b)
        assert torch.equal(whole[0][:, :1, lo:lo + 3], one)


def test_far_positions_and_their_types():
    freqs = serve.frequencies(128, 10000.0)
    f = torch.tensor(freqs, device="cuda")
    q, = random_tensors([(2, 4, 6, 128)], torch.float32, 3, device="cuda")
    for top in (1 << 20, (1 << 31) - 7, 1 << 40):
        pos = np.array([[0, 1, top, top - 1, -top, 12345]] * 2)
        if top < 1 << 31:
            o, none = pa.rope_fwd(q, None, torch.tensor(pos, dtype=torch.int32, device="cuda"), f)
            assert none is None
            _check(o, q, pos, freqs, False, 1.0, False, top)
        o, _ = pa.rope_fwd(q, None, torch.tensor(pos, device="cuda"), f)
        _check(o, q, pos, freqs, False, 1.0, False, top)
        one, _ = pa.rope_fwd(q, None, torch.tensor(pos[0], device="cuda"), f)      # [L]: for every sequence
        assert torch.equal(one, o)


def test_in_place_and_given_outputs():
    f = pa.rope_frequencies(64, device="cuda")
    q, k = random_tensors([(2, 4, 33, 64), (2, 2, 33, 64)], "bf16", 4, device="cuda")
    pos = torch.arange(33, device="cuda", dtype=torch.int32)
    ref = pa.rope_fwd(q, k, pos, f, interleaved=True)
    qo, ko = torch.full_like(q, float("nan")), torch.full_like(k, float("nan"))
    a, b = pa.rope_fwd(q, k, pos, f, qo, ko, interleaved=True)
    assert a is qo and b is ko and torch.equal(qo, ref[0]) and torch.equal(ko, ref[1])
    a, b = pa.rope_fwd(q, k, pos, f, q, k, interleaved=True)
    assert a is q and torch.equal(q, ref[0]) and torch.equal(k, ref[1])


@pytest.mark.parametrize("interleaved", [False, True])
def test_gradient_against_differences(interleaved):
    """The loss sum(g * rope(x)) is linear in x: its difference quotient over a step of
    any size is the gradient up to the rounding of the two losses."""
    rng = np.random.default_rng(5)
    f = pa.rope_frequencies(24, scaling="parts", factor=4.0, original_length=512)
    x, g = rng.standard_normal((2, 2, 3, 5, 32))
    pos = rng.integers(0, 9000, (2, 5))
    dx, _ = pa.rope_bwd(torch.tensor(g, dtype=torch.float32, device="cuda"), None,
                        torch.tensor(pos, device="cuda"), f.cuda(), interleaved=interleaved, magnitude=1.25)
    loss = lambda x: (g * serve.rope(x, pos, f.numpy(), interleaved=interleaved, magnitude=1.25)).sum()   # noqa: E731
    got = host64(dx)
    for i in rng.choice(x.size, 60, replace=False):
        e = np.zeros(x.size)
        e[i] = 1.0
        e = e.reshape(x.shape)
        d = (loss(x + e) - loss(x - e)) / 2
        # g is rounded to 32 bits (2^-24 of two values up to 4.5) beside 6e-7 of the pair
        assert abs(got.reshape(-1)[i] - d) <= 9 * 1.25 * (6e-7 + 2.0 ** -24) + 1e-12, i


def test_streams_and_graph_replays():
    f = pa.rope_frequencies(128, device="cuda")
    q, k = random_tensors([(4, 8, 1, 128), (4, 2, 1, 128)], "f16", 6, device="cuda")
    pos = torch.tensor([[5], [70], [0], [3000]], dtype=torch.int32, device="cuda")
    ref = pa.rope_fwd(q, k, pos, f)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    other = pa.rope_fwd(q, k, pos, f, stream=s)
    s.synchronize()
    assert torch.equal(other[0], ref[0]) and torch.equal(other[1], ref[1])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = pa.rope_fwd(q, k, pos, f)
    for r in range(4):
        pos.fill_(17 * r)
        want = pa.rope_fwd(q, k, pos, f)
        for t in out:
            t.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1]), r


def test_refusals():
    q, k = random_tensors([(2, 4, 3, 64), (2, 2, 3, 64)], "f16", 7, device="cuda")
    f, pos = pa.rope_frequencies(64, device="cuda"), torch.zeros(2, 3, dtype=torch.int32, device="cuda")
    t = q.transpose(1, 2).contiguous().transpose(1, 2)
    x = torch.zeros(q.numel() + 1, dtype=q.dtype, device="cuda")
    bad = [lambda: pa.rope_fwd(q.cpu(), k, pos, f), lambda: pa.rope_fwd(q.double(), None, pos, f),
           lambda: pa.rope_fwd(q, k.float(), pos, f), lambda: pa.rope_fwd(q, k[:1], pos, f),
           lambda: pa.rope_fwd(q, k[:, :, :2], pos, f), lambda: pa.rope_fwd(q, k, pos.float(), f),
           lambda: pa.rope_fwd(q, k, pos[:, :2], f), lambda: pa.rope_fwd(q, k, pos.t(), f),
           lambda: pa.rope_fwd(q, k, pos, f.float()), lambda: pa.rope_fwd(q, k, pos, f.cpu()),
           lambda: pa.rope_fwd(q, k, pos.cpu(), f), lambda: pa.rope_fwd(q, k, pos, f[:0]),
           lambda: pa.rope_fwd(q[0], None, pos, f), lambda: pa.rope_fwd(q.transpose(2, 3), None, pos, f),
           lambda: pa.rope_fwd(q, None, pos, f, k_out=k), lambda: pa.rope_fwd(q, k, pos, f, q[:1]),
           lambda: pa.rope_fwd(q, k, pos, f, q.float()), lambda: pa.rope_fwd(t, None, pos, f, t),
           lambda: pa.rope_fwd(x[:-1].view_as(q), None, pos, f, x[1:].view_as(q)),
           lambda: pa.rope_fwd(q, k, pos, f, x[:q.numel()].view_as(q), x[:k.numel()].view_as(k)),
           lambda: pa.rope_fwd(q, q, pos, f, q), lambda: pa.rope_fwd(q, k, pos, f, k_out=q[:, :2].contiguous()[:, :1]),
           lambda: pa.rope_fwd(q, k, pos, f, magnitude=float("inf")),
           lambda: pa.rope_fwd(q, k, pos, torch.cat((f, f)).contiguous()),
           lambda: pa.rope_fwd(q[:, :, :0], None, pos[:, :0].contiguous(), f)]
    for i, call in enumerate(bad):
        with pytest.raises((ValueError, pa.AttnError)):
            call()
            print("not refused:", i)
