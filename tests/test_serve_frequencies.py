"""rope_frequencies near the ends of 64 bits: finite arguments whose frequencies are not finite, or
vanish because the base overflowed, are refused (no GPU)."""

import math

import pytest

import paper_2510_08726_amd as pa
from oracle import serve


@pytest.mark.parametrize("R,base,kw", [
    (64, 5e-324, {}),                                            # base^(-62 / 64) is over 1e308
    (64, 1e-300, dict(scaling="linear", factor=1e-300)),
    (4, 1e300, dict(scaling="base", factor=1e300)),              # the base is infinite: frequencies 1, 0
    (16, 1e4, dict(scaling="parts", factor=5e-324, original_length=1.0)),
])
def test_refused(R, base, kw):
    with pytest.raises(pa.AttnError) as e:
        pa.rope_frequencies(R, base, **kw)
    assert e.value.status == pa.ATTN_ERR_SHAPE


@pytest.mark.parametrize("R,base,kw", [
    (64, 1e300, {}), (64, 1e-300, {}), (2, 5e-324, {}), (128, 5e5, dict(scaling="base", factor=64.0)),
    (16, 1e4, dict(scaling="parts", factor=1e300, original_length=4096.0)),
])
def test_extreme_but_finite(R, base, kw):
    """Each power, product and quotient in 64 bits is off by a few steps of 2^-52."""
    f = pa.rope_frequencies(R, base, **kw).tolist()
    want = serve.frequencies(R, base, **kw)
    assert all(math.isfinite(x) and abs(x - w) <= 1e-14 * abs(w) for x, w in zip(f, want))
