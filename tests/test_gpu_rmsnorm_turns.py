"""The norms over more rows than workgroups (each takes rows in turn, the next ones' words on their way): every row has the bits
that it has among few, in place too, also where rows share 16-byte words."""

import pytest
import torch

import paper_2510_08726_amd as pa

pytestmark = pytest.mark.gpu

DT = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
TYPES = [("bf16", "bf16"), ("f16", "f32"), ("f32", "f32")]
# Rows of one, two and four steps of a lane, a multiple of 8 long or not; five turns, two and a half, several rows a workgroup.
SIZES = [(1285, 4099), (1024, 4096), (1300, 5119), (643, 8201), (515, 8200), (515, 16393), (9001, 37), (5003, 771)]
FEW = 128                                        # (a multiple of 8: a row's words begin where they did)


def draw(N, M, dtype, wide):
    g = torch.Generator("cuda").manual_seed(N + M)
    t = lambda *s: torch.randn(s, generator=g, device="cuda")     # noqa: E731
    return (t(N, M).to(DT[dtype]), t(N, M).to(DT[wide]), (1 + 0.2 * t(M)).to(DT[dtype]), t(N, M).to(DT[dtype]),
            t(N, M).to(DT[wide]))


def by_few(f, *rows):
    """f of a few rows at a time, its outputs joined."""
    parts = [f(*[r[i:i + FEW] for r in rows]) for i in range(0, len(rows[0]), FEW)]
    return [torch.cat(p) for p in zip(*parts)]


def same(a, b):
    bits = {1: torch.uint8, 2: torch.int16, 4: torch.int32}[a.element_size()]
    return torch.equal(a.contiguous().view(bits), b.contiguous().view(bits))


@pytest.mark.parametrize("N,M", SIZES)
@pytest.mark.parametrize("types", TYPES)
def test_rows_in_turn(N, M, types):
    x, res, w, dy, dh = draw(N, M, *types)
    y, h, rstd = pa.rmsnorm_add(x, res, w)
    few = by_few(lambda a, b: pa.rmsnorm_add(a, b, w), x, res)
    assert all(same(a, b) for a, b in zip((y, h, rstd), few))
    y1, _, rstd1 = pa.rmsnorm_add(x, None, w)
    few = by_few(lambda a: [pa.rmsnorm_add(a, None, w)[i] for i in (0, 2)], x)
    assert same(y1, few[0]) and same(rstd1, few[1])
    a, b = x.clone(), res.clone()
    pa.rmsnorm_add(a, b, w, y=a, h=b)
    assert same(a, y) and same(b, h)
    for dtype, group in ((torch.float8_e4m3fn, 0), (torch.int8, 128)):
        q, s, hq = pa.rmsnorm_add_quant(x, res, w, dtype=dtype, group=group)
        few = by_few(lambda a, b: pa.rmsnorm_add_quant(a, b, w, dtype=dtype, group=group), x, res)
        assert same(q, few[0]) and same(s, few[1]) and same(hq, h)


@pytest.mark.parametrize("N,M", SIZES)
@pytest.mark.parametrize("types", TYPES)
def test_gradients_of_rows_in_turn(N, M, types):
    _, h, w, dy, dh = draw(N, M, *types)
    rstd = h.double().square().mean(-1).rsqrt().float()
    for above in (dh, None):
        dx, dres, dw = pa.rmsnorm_add_bwd(dy, h, rstd, w, above)
        if above is None:
            few = by_few(lambda a, b, c: pa.rmsnorm_add_bwd(a, b, c, w)[:2], dy, h, rstd)
        else:
            few = by_few(lambda a, b, c, d: pa.rmsnorm_add_bwd(a, b, c, w, d)[:2], dy, h, rstd, above)
        assert same(dx, few[0]) and same(dres, few[1])
        # A column's terms: one rounding of n, an fma a row of its workgroup, then the workgroups' (at most 1024 of them, or the
        # rows of one a workgroup): every eighth in turn, eight more, and four rows of a workgroup.
        terms = dy.double() * h.double() * rstd.double()[:, None]
        off = (1 + -(-N // 256) + 1024 / 8 + 8 + 4) * 2.0 ** -24 * terms.abs().sum(0)
        assert bool(((dw.double() - terms.sum(0)).abs() <= off).all())
        again = pa.rmsnorm_add_bwd(dy, h, rstd, w, above)
        assert same(again[0], dx) and same(again[2], dw)
    a, b = dy.clone(), dh.clone()
    one = types[0] == types[1]
    dx, dres, dw = pa.rmsnorm_add_bwd(dy, h, rstd, w, dh)
    got = pa.rmsnorm_add_bwd(a, h, rstd, w, b, dx=a) if one else pa.rmsnorm_add_bwd(a, h, rstd, w, b, dx=a, dresidual=b)
    assert same(got[0], dx) and same(got[1], dres) and same(got[2], dw)


def test_a_matrix_ends_where_its_memory_does():
    """Words at a matrix's ends are read no further than it goes: what lies behind it and before it stays out of the results."""
    for dtype in (torch.bfloat16, torch.float16, torch.float32):
        for N, M in ((1, 1), (3, 5), (1, 7), (2, 13), (3, 1027)):
            big = torch.full((2 * 64 + N * M,), float("nan"), dtype=dtype, device="cuda")
            for lead in (0, 1, 3):
                v = big.clone()
                x = v[64 + lead - 3:64 + lead - 3 + N * M].view(N, M)
                x.copy_(torch.randn(N, M, device="cuda"))
                out = torch.full_like(v, float("nan"))
                y = out[65:65 + N * M].view(N, M)
                want, _, r = pa.rmsnorm_add(x.clone())
                pa.rmsnorm_add(x, None, None, y=y)
                torch.cuda.synchronize()
                assert same(y, want)
                assert bool(out[:65].isnan().all()) and bool(out[65 + N * M:].isnan().all())
                dx, _, dw = pa.rmsnorm_add_bwd(x, x, r, torch.ones(M, dtype=dtype, device="cuda"))
                c = x.clone()
                dx1, _, dw1 = pa.rmsnorm_add_bwd(c, c.clone(), r, torch.ones(M, dtype=dtype, device="cuda"))
                assert same(dx, dx1) and same(dw, dw1) and bool(torch.isfinite(dx).all())


@pytest.mark.parametrize("M", [8192, 4099])
def test_offsets_past_32_bits(M):
    """More than 2^32 bytes and 2^31 elements a matrix: the last rows have the bits that they have alone."""
    N = (2 ** 31 // M // FEW + 2) * FEW
    g = torch.Generator("cuda").manual_seed(M)
    x = torch.empty(N, M, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    w = torch.ones(M, dtype=torch.bfloat16, device="cuda")
    at = slice(N - FEW, N)
    y, h, rstd = pa.rmsnorm_add(x, x, w)
    alone = pa.rmsnorm_add(x[at], x[at], w)
    assert all(same(a[at], b) for a, b in zip((y, h, rstd), alone))
    del y
    q, s, _ = pa.rmsnorm_add_quant(x, None, w)
    alone = pa.rmsnorm_add_quant(x[at], None, w)
    assert same(q[at], alone[0]) and same(s[at], alone[1])
    assert same(pa.quant8_load(q, s)[at], pa.quant8_load(q[at], s[at]))
    del q
    dx, _, dw = pa.rmsnorm_add_bwd(x, h, rstd, w, x)
    assert same(dx[at], pa.rmsnorm_add_bwd(x[at], h[at], rstd[at], w, x[at])[0])
    assert bool(torch.isfinite(dw).all())
    del x, h, dx
    torch.cuda.empty_cache()


@pytest.mark.parametrize("M", [5, 37, 771, 8201])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_row_that_is_not_finite_stays_alone(M, bad):
    """Rows whose elements lie in one 16-byte word with those of a row that is not finite."""
    for dtype in ("bf16", "f32"):
        x, res, w, dy, dh = draw(19, M, dtype, dtype)
        rows = [i for i in range(19) if i != 7]
        good = [*pa.rmsnorm_add(x, res, w), *pa.rmsnorm_add_quant(x, res, w)[:2]]
        rstd = good[2].clone()
        good += pa.rmsnorm_add_bwd(dy, good[1], rstd, w, dh)[:1]
        h = good[1].clone()
        for t in (x, res, dy, dh, h):
            t[7] = bad
        got = [*pa.rmsnorm_add(x, res, w), *pa.rmsnorm_add_quant(x, res, w)[:2], *pa.rmsnorm_add_bwd(dy, h, rstd, w, dh)[:1]]
        assert all(same(a[rows], b[rows]) for a, b in zip(got, good))
        assert bool(got[4][7].isnan().all()) and not bool(torch.isfinite(got[0][7].float()).all())
