"""The operators of a training step around attention: what is timed, and their plain forms.

Attention that keeps its rows' log-sum-exp (``attn_fwd_lse``) and its backward pass
(``attn_bwd``), and the root-mean-square norm with the residual's addition (``rmsnorm_add``),
its backward pass (``rmsnorm_add_bwd``) and its output in 8 bits with scales
(``rmsnorm_add_quant``, read back by ``quant8_load``).  ``run`` computes either the plain form,
in elementary torch operations on 32 bits (64 for what is rounded to 8 bits), or calls the
package, as ``own`` says.  Head counts, head dims, score modifiers and lengths are those of
``paper_2510_08726_amd.workloads``; the other sizes are generic ones: 1 to 16384 rows of 64 to
16384 elements, odd ones among them.
"""

import math

import torch

own = False

_DTYPE = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
_CODE = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}
_TOP = {"e4m3": 448.0, "int8": 127.0}
_EPS = 1e-6


def _attn(name, op, B, Hq, Hkv, Lq, Lk, D, dtype, causal, alibi=False, softcap=0.0, window=0):
    return {"name": name, "op": op, "B": B, "Hq": Hq, "Hkv": Hkv, "Lq": Lq, "Lk": Lk, "D": D, "dtype": dtype,
            "causal": causal, "alibi": alibi, "softcap": softcap, "window": window}


def _norm(name, op, N, M, dtype, stream="", residual=True, offset=0.0):
    return {"name": name, "op": op, "N": N, "M": M, "dtype": dtype, "stream": stream or dtype, "residual": residual,
            "offset": offset}


def _quant(name, N, M, dtype, code, group, residual=True, offset=0.0):
    return {"name": name, "op": "quant", "N": N, "M": M, "dtype": dtype, "stream": dtype, "residual": residual,
            "offset": offset, "code": code, "group": group}


def listed():
    return [
        # The forward pass of a short sequence: latency counts.
        _attn("forward short", "fwd", 1, 12, 12, 127, 127, 64, "f16", True),
        # The forward pass over long sequences with grouped heads.
        _attn("forward long", "fwd", 1, 32, 8, 8192, 8192, 128, "bf16", True),
        # The gradient of one short, unmasked sequence: latency counts.
        _attn("gradient short", "bwd", 1, 8, 8, 128, 128, 64, "f16", False),
        # A batch of ordinary sequences, grouped heads.
        _attn("gradient grouped", "bwd", 2, 32, 8, 2048, 2048, 128, "bf16", True),
        # Odd lengths, more keys than queries, capped scores in a sliding window.
        _attn("gradient window", "bwd", 1, 32, 16, 3001, 4099, 128, "f16", True, softcap=50.0, window=1025),
        # Long sequences, every head with keys of its own: the largest.
        _attn("gradient long", "bwd", 1, 32, 32, 8192, 8192, 128, "bf16", True),
        # One layer's attention in a training step, narrow heads with linear biases.
        _attn("attention step", "step", 2, 16, 16, 2047, 2047, 64, "f16", True, alibi=True),
        # The norm before a layer in a decode step of a few requests: latency counts.
        _norm("norm decode step", "norm", 8, 4096, "bf16"),
        # The norm over a batch of prompts, the residual stream in full precision.
        _norm("norm prompts", "norm", 16384, 4096, "bf16", stream="f32"),
        # The gradient in a training step of odd width.
        _norm("norm gradient", "norm_bwd", 8191, 5119, "bf16", offset=1.0),
        # Activations for an 8-bit product: a scale for each row in a decode step.
        _quant("quant decode step", 16, 5120, "f16", "int8", 0),
        # The same over a batch of prompts, a scale for each 128 elements.
        _quant("quant prompts", 8192, 8192, "bf16", "e4m3", 128),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_HEADS = [(32, 32, 128), (32, 8, 128), (64, 8, 128), (32, 16, 128), (16, 16, 64), (12, 12, 64), (32, 4, 64),
          (40, 2, 128), (7, 1, 64)]


def draw(rng):
    while True:
        op = rng.choice(["fwd", "bwd", "bwd", "bwd", "step", "norm", "norm", "norm_bwd", "norm_bwd", "quant", "quant"])
        dtype = rng.choice(["f16", "bf16"])
        if op in ("fwd", "bwd", "step"):
            Hq, Hkv, D = rng.choice(_HEADS)
            Lq = _log(rng, 1, 8192)
            Lk = max(2, rng.choice([Lq, Lq, _log(rng, 1, 8192)]))    # (one key alone has no gradient but its value's)
            mod = rng.choice(["", "causal", "causal", "causal", "alibi", "causal alibi", "causal softcap",
                              "causal window", "causal window softcap", "causal window alibi"])
            c = _attn("", op, _log(rng, 1, 16), Hq, Hkv, Lq, Lk, D, dtype, "causal" in mod, "alibi" in mod,
                      50.0 if "softcap" in mod else 0.0, _log(rng, 2, 4096) if "window" in mod else 0)
        else:
            dtype = rng.choice(["f16", "bf16", "f32"])
            N, M = rng.choice([1, _log(rng, 1, 16384), _log(rng, 1, 16384)]), _log(rng, 64, 16384)
            M = rng.choice([M, (M + 63) // 64 * 64, (M + 7) // 8 * 8])
            offset, residual = rng.choice([0.0, 0.0, 1.0]), rng.random() < 0.75
            if op == "quant":
                c = _quant("", N, M, dtype, rng.choice(["e4m3", "int8"]), rng.choice([0, 0, 32, 128]), residual, offset)
            else:
                c = _norm("", op, N, M, dtype, rng.choice([dtype, "f32"]) if residual else dtype, residual, offset)
        w = work(c)
        if 0 < w["flops"] <= 1.4e12 and w["bytes"] <= 6.8e8 and _scores(c) <= 32 * 8192 * 8192:
            del c["name"]
            return c


def _scores(c):
    """Scores that the plain form spreads out."""
    return c["B"] * c["Hq"] * c["Lq"] * c["Lk"] if "Lk" in c else 0


def _pairs(c):
    """Visible (query, key) pairs of one head."""
    if not c["causal"]:
        return c["Lq"] * c["Lk"]
    off, W, Lk = c["Lk"] - c["Lq"], c["window"], c["Lk"]
    return sum(max(0, i + off + 1) - (max(0, i + off + 1 - W) if W else 0) for i in range(c["Lq"])) if Lk else 0


def work(case):
    c = case
    if c["op"] in ("fwd", "bwd", "step"):
        q, k, r = 2.0 * c["B"] * c["Hq"] * c["Lq"] * c["D"], 2.0 * c["B"] * c["Hkv"] * c["Lk"] * c["D"], \
            4.0 * c["B"] * c["Hq"] * c["Lq"]
        product = 2.0 * c["B"] * c["Hq"] * c["D"] * _pairs(c)
        fwd = {"bytes": 2 * q + 2 * k + r, "flops": 2 * product}          # q, k, v in; o, lse out
        bwd = {"bytes": 4 * q + 4 * k + r, "flops": 5 * product}          # do, q, k, v, o, lse in; dq, dk, dv out
        if c["op"] == "step":
            return {"bytes": 4 * q + 4 * k + r, "flops": 7 * product}     # do, q, k, v in; o, lse and gradients out
        return fwd if c["op"] == "fwd" else bwd
    n = float(c["N"]) * c["M"]
    e, s = (4.0 if c[t] == "f32" else 2.0 for t in ("dtype", "stream"))
    if c["op"] == "norm":          # x, residual, weight in; y, h, rstd out
        return {"bytes": n * (2 * e + (2 * s if c["residual"] else 0)) + e * c["M"] + 4.0 * c["N"], "flops": 5 * n}
    if c["op"] == "norm_bwd":      # dy, h, dh, rstd, weight in; dx (of both types), dweight out
        return {"bytes": n * (e + 2 * s + (s if c["residual"] else 0) + (e if e != s else 0)) + 4.0 * c["N"]
                + (e + 4) * c["M"], "flops": 11 * n}
    scales = 4.0 * c["N"] * _groups(c)
    # x, residual, weight in; codes, scales, h out; codes and scales in, values out
    return {"bytes": n * (e + (2 * s if c["residual"] else 0) + 1) + e * c["M"] + scales + n * (1 + e) + scales,
            "flops": 9 * n}


def _groups(c):
    return -(-c["M"] // c["group"]) if c["group"] else 1


# What a program has in hand.

def _normal(shape, dtype, g, size=1.0):
    return (size * torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)).to(dtype)


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = _DTYPE[c["dtype"]]
    s = {"case": c}
    if c["op"] in ("fwd", "bwd", "step"):
        gain = 1.0 + 3.0 * (torch.arange(c["D"], device="cuda") % 13 == 5)     # K has a few strong channels
        s["q"] = _normal((c["B"], c["Hq"], c["Lq"], c["D"]), dt, g)
        s["k"] = (_normal((c["B"], c["Hkv"], c["Lk"], c["D"]), torch.float32, g) * gain).to(dt)
        s["v"] = _normal((c["B"], c["Hkv"], c["Lk"], c["D"]), dt, g)
        s["slopes"] = None
        if c["alibi"]:
            s["slopes"] = 2.0 ** (-8.0 * torch.arange(1, c["Hq"] + 1, device="cuda", dtype=torch.float32) / c["Hq"])
        if c["op"] != "fwd":
            # As the layer behind it gives it: a view of [B, Lq, Hq, D], some tokens' losses larger than others'.
            size = torch.exp(_normal((c["B"], c["Lq"], 1, 1), torch.float32, g))
            s["do"] = (_normal((c["B"], c["Lq"], c["Hq"], c["D"]), torch.float32, g) * (0.05 * size)).to(dt).transpose(1, 2)
        if c["op"] == "bwd":
            s["o"], s["lse"] = _forward(s["q"], s["k"], s["v"], s["slopes"], c)
        return s
    N, M, st = c["N"], c["M"], _DTYPE[c["stream"]]
    size = 1.0 + 7.0 * (torch.arange(M, device="cuda") % 97 == 31)             # a few strong channels
    s["weight"] = (1.0 - c["offset"] + _normal((M,), torch.float32, g, 0.2)).to(dt)
    if c["op"] == "norm_bwd":
        s["h"] = (_normal((N, M), torch.float32, g, 3.0) * size).to(st)
        s["dy"] = _normal((N, M), dt, g, 0.05)
        s["dh"] = _normal((N, M), st, g, 0.05) if c["residual"] else None
        s["rstd"] = (s["h"].double().square().mean(-1) + _EPS).rsqrt().float()
        return s
    s["x"] = _normal((N, M), dt, g)
    s["residual"] = (_normal((N, M), torch.float32, g, 3.0) * size).to(st) if c["residual"] else None
    return s


# Plain forms.

def _seen(c, device):
    """Which keys each row sees, [Lq, Lk], or None for all."""
    if not c["causal"]:
        return None
    i = torch.arange(c["Lq"], device=device)[:, None] + (c["Lk"] - c["Lq"])
    j = torch.arange(c["Lk"], device=device)[None]
    seen = j <= i
    return seen & (j > i - c["window"]) if c["window"] else seen


def _scores_of(q, k, slopes, c):
    """Scores [B, Hkv, G Lq, Lk] in 32 bits, masked ones -inf, and the derivative of the cap (or None)."""
    B, Hq, Lq, D = q.shape
    H, Lk = k.shape[1], k.shape[2]
    x = (q.float().reshape(B, H, -1, D) @ k.float().transpose(2, 3)) * D ** -0.5
    slope = None
    if c["softcap"]:
        t = torch.tanh(x / c["softcap"])
        x, slope = c["softcap"] * t, 1.0 - t * t
    x = x.reshape(B, Hq, Lq, Lk)
    if slopes is not None:
        i = torch.arange(Lq, device=q.device)[:, None] + (Lk - Lq)
        x = x - slopes[:, None, None] * (i - torch.arange(Lk, device=q.device)[None]).float()
    seen = _seen(c, q.device)
    if seen is not None:
        x = torch.where(seen, x, -math.inf)
    return x.reshape(B, H, -1, Lk), slope


def _forward(q, k, v, slopes, c):
    x, _ = _scores_of(q, k, slopes, c)
    top = x.amax(-1, keepdim=True)
    w = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
    total = w.sum(-1, keepdim=True)
    o = torch.where(total > 0, (w @ v.float()) / total, 0.0)
    return o.reshape(q.shape).to(q.dtype), (top + torch.log(total)).reshape(q.shape[:3])


def _backward(do, q, k, v, o, lse, slopes, c):
    B, H, _, D = k.shape
    x, slope = _scores_of(q, k, slopes, c)
    rows = lambda t: t.float().reshape(B, H, -1, D)     # noqa: E731
    none = (lse == -math.inf).reshape(B, H, -1, 1)
    p = torch.where(none, 0.0, torch.exp(x - lse.reshape(B, H, -1, 1)))
    dv = p.transpose(2, 3) @ rows(do)
    ds = p * (rows(do) @ v.float().transpose(2, 3) - (rows(do) * rows(o)).sum(-1, keepdim=True))
    ds = (ds if slope is None else ds * slope) * D ** -0.5
    dq, dk = ds @ k.float(), ds.transpose(2, 3) @ rows(q)
    return dq.reshape(q.shape).to(q.dtype), dk.to(k.dtype), dv.to(v.dtype)


def _add(x, residual):
    return x if residual is None else (x.float() + residual.float()).to(residual.dtype)


def _rmsnorm(x, residual, weight, offset):
    h = _add(x, residual)
    y = h.float()
    rstd = (y.square().mean(-1) + _EPS).rsqrt()
    return (y * rstd[:, None] * (weight.float() + offset)).to(x.dtype), h, rstd


def _rmsnorm_bwd(dy, h, rstd, weight, dh, offset):
    n = h.float() * rstd[:, None]
    g = dy.float() * (weight.float() + offset)
    dx = rstd[:, None] * (g - n * (g * n).mean(-1, keepdim=True))
    if dh is not None:
        dx = dx + dh.float()
    return dx.to(dy.dtype), dx.to(h.dtype), (dy.float() * n).sum(0)


def _pad_groups(y, c):
    """y [N, M] as [N, groups, group], zeros behind the last element."""
    G = _groups(c)
    n = c["group"] or c["M"]
    return torch.nn.functional.pad(y, (0, G * n - c["M"])).reshape(-1, G, n)


def _rmsnorm_quant(x, residual, weight, c):
    h = _add(x, residual)
    y = h.double()
    y = y * (y.square().mean(-1, keepdim=True) + _EPS).rsqrt() * (weight.double() + c["offset"])
    z = _pad_groups(y, c)
    scale = (z.abs().amax(-1, keepdim=True) / _TOP[c["code"]]).float()
    z = torch.where(scale > 0, z / scale.double(), 0.0)
    if c["code"] == "int8":
        z = z.round()
    else:
        # Three bits behind the leading one, down to multiples of 2^-9; ties to the even code.
        step = torch.ldexp(torch.ones((), dtype=torch.float64, device=z.device), (torch.frexp(z)[1] - 4).clamp(min=-9))
        z = (z / step).round() * step
    values = (z.float() * scale).flatten(1)[:, :c["M"]].to(x.dtype)
    return values, scale[..., 0], h


def run(state):
    s, c = state, state["case"]
    op = c["op"]
    if own:
        return _run_own(s, c, op)
    if op == "norm":
        return _rmsnorm(s["x"], s["residual"], s["weight"], c["offset"])
    if op == "norm_bwd":
        return _rmsnorm_bwd(s["dy"], s["h"], s["rstd"], s["weight"], s["dh"], c["offset"])
    if op == "quant":
        return _rmsnorm_quant(s["x"], s["residual"], s["weight"], c)
    if op == "bwd":
        return _backward(s["do"], s["q"], s["k"], s["v"], s["o"], s["lse"], s["slopes"], c)
    o, lse = _forward(s["q"], s["k"], s["v"], s["slopes"], c)
    if op == "fwd":
        return o, lse
    return (o, lse, *_backward(s["do"], s["q"], s["k"], s["v"], o, lse, s["slopes"], c))


def _run_own(s, c, op):
    import paper_2510_08726_amd as pa
    if op == "norm":
        return pa.rmsnorm_add(s["x"], s["residual"], s["weight"], eps=_EPS, weight_offset=c["offset"])
    if op == "norm_bwd":
        return pa.rmsnorm_add_bwd(s["dy"], s["h"], s["rstd"], s["weight"], s["dh"], weight_offset=c["offset"])
    if op == "quant":
        q, scales, h = pa.rmsnorm_add_quant(s["x"], s["residual"], s["weight"], dtype=_CODE[c["code"]],
                                            group=c["group"], eps=_EPS, weight_offset=c["offset"])
        return pa.quant8_load(q, scales, group=c["group"], dtype=s["x"].dtype), scales, h
    how = {"causal": c["causal"], "alibi_slopes": s["slopes"], "softcap": c["softcap"] or None,
           "window": c["window"] or None}
    if op == "bwd":
        return pa.attn_bwd(s["do"], s["q"], s["k"], s["v"], s["o"], s["lse"], **how)
    o, lse = pa.attn_fwd_lse(s["q"], s["k"], s["v"], **how)
    if op == "fwd":
        return o, lse
    return (o, lse, *pa.attn_bwd(s["do"], s["q"], s["k"], s["v"], o, lse, **how))


# The definitions in 64 bits, apart from the plain forms.

def _attention64(s, c):
    """o, lse and the gradients of q, k and v, head by head: the derivative of softmax(s) v itself,
    which takes neither o nor lse from the state."""
    q, k, v = (s[t].double() for t in ("q", "k", "v"))
    do = s["do"].double() if "do" in s else None
    G, Lq, Lk = c["Hq"] // c["Hkv"], c["Lq"], c["Lk"]
    o, lse, dq = torch.zeros_like(q), torch.zeros(q.shape[:3], dtype=torch.float64, device=q.device), torch.zeros_like(q)
    dk, dv = torch.zeros_like(k), torch.zeros_like(v)
    ahead = (torch.arange(Lk - Lq, Lk, device=q.device)[:, None] - torch.arange(Lk, device=q.device)[None])
    hidden = torch.zeros_like(ahead, dtype=torch.bool)
    if c["causal"]:
        hidden = (ahead < 0) | (ahead >= c["window"]) if c["window"] else ahead < 0
    blind = hidden.all(-1, keepdim=True)
    for b in range(c["B"]):
        for hq in range(c["Hq"]):
            h = hq // G
            raw = torch.mm(q[b, hq], k[b, h].t().contiguous()) / math.sqrt(c["D"])
            x = c["softcap"] * torch.tanh(raw / c["softcap"]) if c["softcap"] else raw
            if s["slopes"] is not None:
                x = x - s["slopes"][hq].double() * ahead
            x = x.masked_fill(hidden, -math.inf)
            lse[b, hq] = torch.logsumexp(x, -1)
            p = torch.softmax(x, -1).masked_fill(blind, 0.0)
            o[b, hq] = torch.mm(p, v[b, h])
            if do is None:
                continue
            g = do[b, hq].contiguous()
            dv[b, h] += torch.mm(p.t().contiguous(), g)
            d = torch.mm(g, v[b, h].t().contiguous())
            d = p * (d - (p * d).sum(-1, keepdim=True)) / math.sqrt(c["D"])
            if c["softcap"]:
                d = d / torch.cosh(raw / c["softcap"]).square()
            dq[b, hq] = torch.mm(d, k[b, h])
            dk[b, h] += torch.mm(d.t().contiguous(), q[b, hq])
    return o, lse, dq, dk, dv


def _eighth64(z, code):
    """The nearest values of a grid of 8-bit codes, ties to the even code: by looking them up."""
    if code == "int8":
        grid = torch.arange(128, dtype=torch.float64, device=z.device)
    else:
        n = torch.arange(127, device=z.device)
        e, m = (n >> 3).double(), (n & 7).double()
        grid = torch.where(e > 0, (8 + m) * 2.0 ** (e - 10), m * 2.0 ** -9)
    a = z.abs()
    at = torch.bucketize(a, (grid[1:] + grid[:-1]) / 2)             # the first middle that is not under a
    tie = a == ((grid[1:] + grid[:-1]) / 2)[at.clamp(max=len(grid) - 2)]
    at = at + (tie & (at % 2 == 1)).long()                          # between at and at + 1: the even one
    return grid[at.clamp(max=len(grid) - 1)] * z.sign()


def exact(case, seed):
    c = case
    s = prepare(case, seed)
    if c["op"] in ("fwd", "bwd", "step"):
        got = _attention64(s, c)
        return {"fwd": got[:2], "bwd": got[2:], "step": got}[c["op"]]
    w = s["weight"].double() + c["offset"]
    if c["op"] == "norm_bwd":
        h, r, dy = s["h"].double(), s["rstd"].double()[:, None], s["dy"].double()
        inner = (dy * w * h).sum(-1, keepdim=True) / c["M"]
        dx = r * w * dy - r ** 3 * h * inner
        if s["dh"] is not None:
            dx = dx + s["dh"].double()
        return dx, dx, (dy * h * r).sum(0)
    x = s["x"].double()
    h = x
    if s["residual"] is not None:
        h = (x + s["residual"].double()).to(s["residual"].dtype).double()    # what is kept is what is normed
    rstd = 1.0 / torch.sqrt((h * h).sum(-1) / c["M"] + _EPS)
    y = h * w * rstd[:, None]
    if c["op"] == "norm":
        return y, h, rstd
    n = c["group"] or c["M"]
    values, scales = torch.empty_like(y), []
    for a in range(0, c["M"], n):
        part = y[:, a:a + n]
        scale = (part.abs().max(-1).values / _TOP[c["code"]]).float().double()
        values[:, a:a + n] = _eighth64(part / scale[:, None].clamp(min=1e-300), c["code"]) * scale[:, None]
        scales.append(scale)
    return values, torch.stack(scales, -1), h
