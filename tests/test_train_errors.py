"""The check of attention's errors in training as root mean squares finds what it is for: mistakes planted in the emulated
kernels (no GPU)."""

import pytest

import train_errors as te

NAMES = ("o", "lse", "dq", "dk", "dv")


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("case", te.CASES)
@pytest.mark.parametrize("mutant,outputs", [(dict(dq_once=True), ["dq"]), (dict(drop=2), ["dq", "dk"]), (dict(drop=4), ["dq", "dk"]),
                                            (dict(exponent=2.0 ** -7), ["dv", "dk"])], ids=str)
def test_a_rounding_too_many_is_found(case, dtype, mutant, outputs):
    x = te.inputs(case, dtype)
    want, plain = te.both64(case, x, dtype)
    _, off = te.both64(case, x, dtype, **mutant)
    assert all(v == 1.0 for v in te.shares({n: plain[n] for n in NAMES}, want, plain).values())
    got = te.shares({n: off[n] for n in NAMES}, want, plain)
    assert all(got[n] > te.MORE for n in outputs), got


@pytest.mark.parametrize("case", te.FAR[1:3])
def test_exponents_rounded_beside_a_large_bias_are_found(case):
    """2^-24 of 2^13, several times."""
    x = te.inputs(case, "f16")
    want, plain = te.both64(case, x, "f16")
    _, off = te.both64(case, x, "f16", exponent=2.0 ** -10)
    assert te.shares({"dv": off["dv"]}, want, plain)["dv"] > te.MORE
