"""The operators of a training step as programs call them: outputs and workspaces of the caller's, both Python paths,
streams, graphs, two calls at once, extreme values, and a block of them together."""

import math

import numpy as np
import pytest
import torch

import paper_2510_08726_amd as pa
from train_cases import bounds, check, draw, oracle64

pytestmark = pytest.mark.gpu


def _attn(seed=1, dtype="bf16", B=2, Hq=8, Hkv=2, L=300, D=128):
    do, q, k, v, _ = [None if t is None else t.cuda() for t in draw(B, Hq, Hkv, L, L, D, dtype, seed)]
    return do.transpose(1, 2).contiguous().transpose(1, 2), q, k, v


def _norm(seed=1, N=300, M=1000, dtype=torch.bfloat16, wide=torch.float32):
    g = torch.Generator().manual_seed(seed)
    t = lambda *s: torch.randn(s, generator=g)     # noqa: E731
    return [x.cuda() for x in (t(N, M).to(dtype), t(N, M).to(wide), t(M).to(dtype), t(N, M).to(dtype), t(N, M).to(wide))]


def _calls(seed=1, **kw):
    """Name -> a call that takes keyword arguments, its outputs' names, and its workspace's size or None."""
    do, q, k, v = _attn(seed, **kw)
    x, res, w, dy, dh = _norm(seed)
    how = dict(causal=True, softcap=30.0, window=100)
    o, lse = pa.attn_fwd_lse(q, k, v, **how)
    y, h, rstd = pa.rmsnorm_add(x, res, w)
    codes, scales, _ = pa.rmsnorm_add_quant(x, res, w, group=64)
    B, Hq, L, D = q.shape
    return {
        "fwd": (lambda **a: pa.attn_fwd_lse(q, k, v, **how, **a), ("o", "lse"), None),
        "bwd": (lambda **a: pa.attn_bwd(do, q, k, v, o, lse, **how, **a), ("dq", "dk", "dv"),
                pa.attn_bwd_workspace_bytes(B, Hq, k.shape[1], L, L, D, True, 100)),
        "norm": (lambda **a: pa.rmsnorm_add(x, res, w, **a), ("y", "h", "rstd"), None),
        "quant": (lambda **a: pa.rmsnorm_add_quant(x, res, w, group=64, **a), ("q", "scales", "h"), None),
        "load": (lambda **a: pa.quant8_load(codes, scales, group=64, **a), ("y",), None),
        "norm_bwd": (lambda **a: pa.rmsnorm_add_bwd(dy, h, rstd, w, dh, **a), ("dx", "dresidual", "dweight"),
                     pa.rmsnorm_add_bwd_workspace_bytes(*x.shape)),
    }


def _tuple(r):
    return r if isinstance(r, tuple) else (r,)


def _same(a, b):
    return all(torch.equal(x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x,
                           y.view(torch.uint8) if y.dtype == torch.float8_e4m3fn else y) for x, y in zip(a, b))


NAMES = ["fwd", "bwd", "norm", "quant", "load", "norm_bwd"]


@pytest.mark.parametrize("name", NAMES)
def test_given_outputs_workspace_and_both_paths(monkeypatch, name):
    call, outs, size = _calls()[name]
    ref = [t.clone() for t in _tuple(call())]
    for path in ("marshalled", "checked"):
        if path == "checked":
            monkeypatch.setattr(pa, "_BINDING", pa._NotBuilt)
        assert _same(_tuple(call()), ref), path
        given = {n: torch.full_like(t, 3) if t.dtype != torch.float8_e4m3fn else torch.empty_like(t) for n, t in zip(outs, ref)}
        ws = {} if size is None else {"workspace": torch.full((size,), 255, dtype=torch.uint8, device="cuda")}
        got = _tuple(call(**given, **ws))
        assert all(a is given[n] for a, n in zip(got, outs)) and _same(got, ref), path
        if ws:
            with pytest.raises(pa.AttnError):
                call(workspace=torch.empty(size - 1, dtype=torch.uint8, device="cuda"))
        for n, t in zip(outs, ref):          # of another shape, type or place
            for bad in (t[..., :-1], t.double() if t.dtype != torch.float8_e4m3fn else t.float(), t.cpu(), t[None]):
                with pytest.raises(ValueError):
                    call(**{n: bad})


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("path", ["marshalled", "checked"])
def test_on_a_given_stream(monkeypatch, name, path):
    call, _, _ = _calls()[name]
    ref = [t.clone() for t in _tuple(call())]
    if path == "checked":
        monkeypatch.setattr(pa, "_BINDING", pa._NotBuilt)
    s = torch.cuda.Stream()
    for r in range(4):
        s.wait_stream(torch.cuda.current_stream())
        got = _tuple(call(stream=s))
        torch.cuda.current_stream().wait_stream(s)
        assert _same(got, ref), r
        for t in got:
            t.record_stream(torch.cuda.current_stream())


def test_two_calls_at_once():
    """Each with a workspace of its own, on streams of their own."""
    a, b = _calls(1), _calls(2, dtype="f16", D=64, Hkv=8)
    for name in NAMES:
        want = [[t.clone() for t in _tuple(c[name][0]())] for c in (a, b)]
        streams = [torch.cuda.Stream(), torch.cuda.Stream()]
        torch.cuda.synchronize()
        for r in range(5):
            got = []
            for c, s in zip((a, b), streams):
                with torch.cuda.stream(s):
                    got.append(_tuple(c[name][0]()))
            torch.cuda.synchronize()
            assert all(_same(g, w) for g, w in zip(got, want)), (name, r)


def test_graphs():
    """Captured, and replayed with eager work on other data between: two graphs beside each other, whose workspaces come
    from one pool."""
    calls = _calls(3)
    ref = {n: [t.clone() for t in _tuple(calls[n][0]())] for n in NAMES}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for n in NAMES:
            calls[n][0]()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graphs, outs = [], []
    for names in (NAMES, ["bwd", "norm_bwd"]):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, pool=graphs[0].pool() if graphs else None):
            outs.append({n: _tuple(calls[n][0]()) for n in names})
        graphs.append(g)
    other = _calls(4)
    for r in range(4):
        for g, out in zip(graphs, outs):
            g.replay()
            torch.cuda.synchronize()
            assert all(_same(out[n], ref[n]) for n in out), r
            for n in NAMES:
                other[n][0]()
            torch.cuda.synchronize()


def test_the_same_bits_each_time():
    for kw in (dict(), dict(B=1, Hq=40, Hkv=2, L=1500), dict(B=1, Hq=8, Hkv=8, L=1024, D=64, dtype="f16")):
        do, q, k, v = _attn(5, **kw)
        o, lse = pa.attn_fwd_lse(q, k, v, causal=True)
        ref = pa.attn_bwd(do, q, k, v, o, lse, causal=True)
        for _ in range(10):
            assert _same(pa.attn_bwd(do, q, k, v, o, lse, causal=True), ref)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("scale", [-0.2, 0.0, 1e-6, 1.0])
def test_scales(dtype, scale):
    x = draw(1, 4, 2, 70, 130, 64, dtype, 7)
    for how in (dict(causal=True), dict(causal=True, softcap=4.0), dict()):
        how["scale"] = scale
        r = oracle64(*x, **how)
        d, q, k, v = [t.cuda() for t in x[:4]]
        o, lse = pa.attn_fwd_lse(q, k, v, **how)
        dq, dk, dv = pa.attn_bwd(d, q, k, v, o, lse, **how)
        check({"o": o, "lse": lse, "dq": dq, "dk": dk, "dv": dv}, r, bounds(r, dtype, None, how.get("softcap"), 130), str(how))


@pytest.mark.parametrize("size", [1e-6, 1e-3, 30.0, 3000.0])
def test_gradients_of_any_size_in_fp16(size):
    """What is small in fp16 (weights of long rows, a gradient under no loss scale) keeps its mantissa."""
    x = draw(1, 2, 1, 700, 700, 64, "f16", 9, size=size)
    r = oracle64(*x, causal=True)
    d, q, k, v = [t.cuda() for t in x[:4]]
    o, lse = pa.attn_fwd_lse(q, k, v, causal=True)
    dq, dk, dv = pa.attn_bwd(d, q, k, v, o, lse, causal=True)
    check({"dq": dq, "dk": dk, "dv": dv}, r, bounds(r, "f16"), f"size {size}")


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_zero_gradients_and_large_caps(dtype):
    x = draw(1, 2, 2, 90, 90, 128, dtype, 11)
    d, q, k, v = [t.cuda() for t in x[:4]]
    o, lse = pa.attn_fwd_lse(q, k, v, causal=True)
    for t in pa.attn_bwd(torch.zeros_like(d), q, k, v, o, lse, causal=True):
        assert (t == 0).all()
    how = dict(causal=True, softcap=1024.0)
    r = oracle64(*x, **how)
    o, lse = pa.attn_fwd_lse(q, k, v, **how)
    dq, dk, dv = pa.attn_bwd(d, q, k, v, o, lse, **how)
    check({"lse": lse, "dq": dq, "dk": dk, "dv": dv}, r, bounds(r, dtype, None, 1024.0), "cap 1024")


def test_rows_that_see_nothing():
    """Their gradient's rows are not read (NaN here), their dq is zero, their lse -inf."""
    for window in (None, 5):
        do, q, k, v, _ = draw(2, 2, 1, 150, 60, 64, "bf16", 13)
        do[:, :, :90] = float("nan")
        r = oracle64(do, q, k, v, None, causal=True, window=window)
        d, q, k, v = [t.cuda() for t in (do, q, k, v)]
        o, lse = pa.attn_fwd_lse(q, k, v, causal=True, window=window)
        got = pa.attn_bwd(d, q, k, v, o, lse, causal=True, window=window)
        assert (lse[:, :, :90] == -math.inf).all() and (o[:, :, :90] == 0).all() and (got[0][:, :, :90] == 0).all()
        check(dict(zip(("dq", "dk", "dv"), got)), r, bounds(r, "bf16"), "empty rows")


def test_strides_of_the_gradient():
    """Views of [B, L, H, D], of a part of a wider projection, of one row for all (strides of 0), and one that has to be refused."""
    do, q, k, v, _ = [None if t is None else t.cuda() for t in draw(2, 4, 2, 65, 65, 64, "bf16", 15)]
    o, lse = pa.attn_fwd_lse(q, k, v, causal=True)
    ref = pa.attn_bwd(do, q, k, v, o, lse, causal=True)
    wide = torch.full((2, 65, 3, 4, 64), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, :, 1] = do.transpose(1, 2)
    assert _same(pa.attn_bwd(wide[:, :, 1].transpose(1, 2), q, k, v, o, lse, causal=True), ref)
    assert _same(pa.attn_bwd(do.transpose(1, 2).contiguous().transpose(1, 2), q, k, v, o, lse, causal=True), ref)
    for view in (do[:, :, :1].expand(-1, -1, 65, -1), do[:1, :1].expand(2, 4, -1, -1)):
        assert _same(pa.attn_bwd(view, q, k, v, o, lse, causal=True),
                     pa.attn_bwd(view.contiguous(), q, k, v, o, lse, causal=True))
    for bad in (do.transpose(2, 3).contiguous().transpose(2, 3), do[..., :1].expand(-1, -1, -1, 64)):
        with pytest.raises(ValueError):
            pa.attn_bwd(bad, q, k, v, o, lse, causal=True)
    odd = torch.empty(do.numel() + 1, dtype=torch.bfloat16, device="cuda")[1:].view_as(do).copy_(do)
    with pytest.raises(pa.AttnError):
        pa.attn_bwd(odd, q, k, v, o, lse, causal=True)
    with pytest.raises(pa.AttnError):
        pa.attn_bwd(do, q, k, v, o, lse, dq=do, causal=True)


def test_many_heads_past_2_31_elements():
    """8200 heads of 2048 rows, 2.1e9 elements a tensor: the last heads give what they give alone."""
    H, L, D, W = 8200, 2048, 128, 16
    one = [t.cuda() for t in draw(1, 3, 3, L, L, D, "bf16", 17)[:4]]
    many = [t.expand(1, 3, L, D).repeat(1, H // 3 + 1, 1, 1)[:, -H:].contiguous() for t in one]
    how = dict(causal=True, window=W)
    o, lse = pa.attn_fwd_lse(*many[1:], **how)
    got = (o, lse, *pa.attn_bwd(*many, o, lse, **how))
    assert got[0].numel() > 2 ** 31
    r = oracle64(*[t.cpu() for t in one], None, **how)
    b = bounds(r, "bf16")
    for at in (slice(H - 3, H), slice(1, 4)):       # (head 0 is the third of them)
        check({n: t[:, at] for n, t in zip(("o", "lse", "dq", "dk", "dv"), got)}, r, b, str(at))


def test_norm_past_2_31_elements():
    N, M = 1 << 20, 2056
    x = torch.randn(64, M, device="cuda").to(torch.bfloat16)
    w = torch.randn(M, device="cuda").to(torch.bfloat16)
    big = x.repeat(N // 64, 1)
    assert big.numel() > 2 ** 31
    y, h, rstd = pa.rmsnorm_add(big, None, w)
    ref, _, r = pa.rmsnorm_add(x, None, w)
    assert torch.equal(y[-64:], ref) and torch.equal(rstd[-64:], r) and torch.equal(y[:64], ref)
    del y
    dx, _, dw = pa.rmsnorm_add_bwd(big, big, rstd, w)
    ref, _, dw1 = pa.rmsnorm_add_bwd(x, x, r, w)
    assert torch.equal(dx[-64:], ref) and torch.equal(dx[:64], ref)
    # (16384 times the sum of 64 rows: sums of 2^20 positive-and-negative products in fp32, at most 2^14 one after another)
    size = (x.double() ** 2 * r.double()[:, None]).sum(0) * (N // 64)
    assert ((dw.double() - dw1.double() * (N // 64)).abs() <= 2.0 ** -24 * 2.0 ** 14 * size).all()
    del dx
    q, s, _ = pa.rmsnorm_add_quant(big, None, w, group=128)
    q1, s1, _ = pa.rmsnorm_add_quant(x, None, w, group=128)
    assert torch.equal(q[-64:].view(torch.uint8), q1.view(torch.uint8)) and torch.equal(s[-64:], s1)
    assert torch.equal(pa.quant8_load(q, s, group=128)[-64:], pa.quant8_load(q1, s1, group=128))


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M", [64, 259, 1000])
def test_norm_in_place(dtype, M):
    for wide in {dtype, torch.float32}:
        x, res, w, dy, dh = _norm(7, 37, M, dtype, wide)
        y, h, rstd = pa.rmsnorm_add(x, res, w)
        x2, r2 = x.clone(), res.clone()
        got = pa.rmsnorm_add(x2, r2, w, y=x2, h=r2)
        assert got[0] is x2 and got[1] is r2 and _same(got, (y, h, rstd))
        q = pa.rmsnorm_add_quant(x, res, w, group=32)
        r2 = res.clone()
        assert _same(pa.rmsnorm_add_quant(x, r2, w, h=r2, group=32), q)
        ref = pa.rmsnorm_add_bwd(dy, h, rstd, w, dh)
        d2, h2 = dy.clone(), dh.clone()
        kw = {} if wide == dtype else {"dresidual": h2}
        assert _same(pa.rmsnorm_add_bwd(d2, h, rstd, w, h2, dx=d2, **kw), ref)
        if wide == dtype:
            h2 = dh.clone()
            assert _same(pa.rmsnorm_add_bwd(dy, h, rstd, w, h2, dx=h2), ref)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("code", [torch.int8, torch.float8_e4m3fn])
def test_infinities_zeros_and_extremes_in_8_bits(dtype, code):
    M = 300
    x = torch.ones(7, M, device="cuda", dtype=dtype)
    x[0] = 0
    x[1, 5] = math.inf
    x[2, 299] = math.nan
    x[3, :128] = 0
    x[4] = 1e30
    x[5] = 1e-30
    w = torch.ones(M, device="cuda", dtype=dtype)
    q, s, _ = pa.rmsnorm_add_quant(x, None, w, dtype=code, group=128, eps=1e-6)
    back = pa.quant8_load(q, s, group=128, dtype=torch.float32)
    assert s.shape == (7, 3)
    assert (s[0] == 0).all() and (back[0] == 0).all()
    assert s[1].isnan().tolist() == [True, False, False] and (back[1, 128:] == 0).all() and back[1, :128].isnan().all()
    assert s[2].isnan().all() and back[2].isnan().all()                     # (the row's rstd is NaN)
    assert s[3, 0] == 0 and (back[3, :128] == 0).all() and (back[3, 128:] > 0).all()
    assert (back[4] - 1).abs().max() <= 1e-5                                # squares past the range of 32 bits
    assert back[5].isfinite().all()                                         # eps is all there is under the root: 1e-27
    w[200] = math.nan
    q, s, _ = pa.rmsnorm_add_quant(x[6:], None, w, dtype=code, group=128)
    assert s.isnan().tolist() == [[False, True, False]] and (q.view(torch.uint8)[0, 128:256] == 0).all()
    q, s, _ = pa.rmsnorm_add_quant(x[6:], None, w, dtype=code)
    assert s.isnan().all() and (q.view(torch.uint8) == 0).all()
    y, _, rstd = pa.rmsnorm_add(x, None, None, eps=0.0)
    assert rstd[0] == math.inf and y[0].isnan().all() and (y[4] - 1).abs().max() <= 2.0 ** -8


def test_leading_dims_and_refusals():
    x = torch.randn(2, 3, 5, 64, device="cuda")
    w = torch.randn(64, device="cuda")
    y, h, rstd = pa.rmsnorm_add(x, None, w)
    assert h is x and rstd.shape == (2, 3, 5)
    assert torch.equal(y.view(30, 64), pa.rmsnorm_add(x.view(30, 64), None, w)[0])
    assert pa.rmsnorm_add(x[0, 0, 0])[2].shape == ()
    q, s, _ = pa.rmsnorm_add_quant(x, None, w, group=32)
    assert s.shape == (2, 3, 5, 2) and pa.quant8_load(q, s, group=32).shape == x.shape
    dx, dr, dw = pa.rmsnorm_add_bwd(x, x, rstd, w)
    assert dx.shape == x.shape and dr is dx and dw.shape == (64,)
    for call in (lambda: pa.rmsnorm_add(x.transpose(0, 1)), lambda: pa.rmsnorm_add(x, x.half()), lambda: pa.rmsnorm_add(x, None, w.half()),
                 lambda: pa.rmsnorm_add(x, None, w[:32]), lambda: pa.rmsnorm_add(x.double()), lambda: pa.rmsnorm_add(x, None, w, h=x),
                 lambda: pa.rmsnorm_add(x[:0]), lambda: pa.rmsnorm_add_quant(x, group=48),
                 lambda: pa.rmsnorm_add_quant(x, dtype=torch.uint8), lambda: pa.quant8_load(q, s), lambda: pa.quant8_load(q, s, group=32, dtype=torch.int8),
                 lambda: pa.rmsnorm_add_bwd(x, x, rstd, w, dresidual=x.clone()), lambda: pa.rmsnorm_add_bwd(x, x, rstd, dweight=w),
                 lambda: pa.rmsnorm_add_bwd(x, x.half(), rstd), lambda: pa.rmsnorm_add_bwd(x, x, rstd[0])):
        with pytest.raises(ValueError):
            call()
    big = torch.zeros(1, 32769, device="cuda")
    for call in (lambda: pa.rmsnorm_add(big), lambda: pa.rmsnorm_add(x, x.clone(), w, y=h, h=h)):
        with pytest.raises(pa.AttnError):
            call()


def test_a_block_of_them_together():
    """A layer's attention block, forward and backward, as a program chains the operators, against autograd in 64 bits."""
    B, L, H, Hkv, D = 2, 90, 4, 2, 64
    M, dt = H * D, torch.bfloat16
    g = torch.Generator().manual_seed(19)
    t = lambda *s, size=1.0: (size * torch.randn(s, generator=g)).to(dt)     # noqa: E731
    x, res, w, dy, dres = t(B, L, M), t(B, L, M).float(), (1 + 0.1 * t(M).float()).to(dt), t(B, L, M), t(B, L, M).float()
    wq, wkv = t(M, M, size=M ** -0.5), t(M, 2 * Hkv * D, size=M ** -0.5)
    f = pa.rope_frequencies(D)
    pos = torch.arange(L, dtype=torch.int32)

    c = [a.cuda() for a in (x, res, w, wq, wkv, dy, dres, f, pos)]
    gx, gres, gw, gwq, gwkv, gdy, gdres, gf, gpos = c
    y, h, rstd = pa.rmsnorm_add(gx, gres, gw)
    q = (y.view(-1, M) @ gwq).view(B, L, H, D).transpose(1, 2)
    kv = (y.view(-1, M) @ gwkv).view(B, L, 2, Hkv, D)
    k, v = kv[:, :, 0].transpose(1, 2), kv[:, :, 1].transpose(1, 2).contiguous()
    q, k = pa.rope_fwd(q, k, gpos, gf)
    o, lse = pa.attn_fwd_lse(q, k, v, causal=True)
    dq, dk, dv = pa.attn_bwd(gdy.view(B, L, H, D).transpose(1, 2), q, k, v, o, lse, causal=True)
    dq, dk = pa.rope_bwd(dq, dk, gpos, gf)
    back = lambda a: a.transpose(1, 2).reshape(B * L, -1)     # noqa: E731
    dkv = torch.cat((back(dk), back(dv)), 1)
    d = (back(dq) @ gwq.t().contiguous() + dkv @ gwkv.t().contiguous()).view(B, L, M)
    dx, dr, dw = pa.rmsnorm_add_bwd(d, h, rstd, gw, gdres)

    X, R, W = [a.double().requires_grad_() for a in (x, res, w)]
    Hh = X + R
    Y = Hh * (Hh.square().mean(-1, keepdim=True) + 1e-6).rsqrt() * W
    split = lambda a, n: a.view(B, L, n, D).transpose(1, 2)     # noqa: E731
    Q, KV = split(Y @ wq.double(), H), (Y @ wkv.double()).view(B, L, 2, Hkv, D)
    K, V = KV[:, :, 0].transpose(1, 2), KV[:, :, 1].transpose(1, 2)
    angle = pos.double()[:, None] * f

    def turn(a):
        u, z = a[..., :D // 2], a[..., D // 2:]
        return torch.cat((u * angle.cos() - z * angle.sin(), u * angle.sin() + z * angle.cos()), -1)

    s = turn(Q).view(B, Hkv, H // Hkv, L, D) @ turn(K)[:, :, None].transpose(-1, -2) / math.sqrt(D)
    p = torch.softmax(s.masked_fill(torch.ones(L, L).triu(1).bool(), -math.inf), -1)
    O = (p @ V[:, :, None]).reshape(B, H, L, D)     # noqa: E741
    ((O * split(dy.double(), H)).sum() + (Hh * dres.double()).sum()).backward()
    # Eleven tensors are rounded to bf16 on the way (2^-9 each, of their norm), and the products' operands.
    for name, a, b in (("o", o, O), ("dx", dx, X.grad), ("dresidual", dr, R.grad), ("dweight", dw, W.grad)):
        off = float((a.double().cpu() - b.detach()).norm() / b.detach().norm())
        print(f"{name}: off by {off:.2e}", flush=True)
        assert off <= 11 * 2.0 ** -9, name
    assert dr.dtype == torch.float32 and torch.equal(dr.to(dt), dx)
    assert np.isfinite(lse.cpu().numpy()).all()
