"""attn_fwd_lse takes the tensors that attn_bwd takes: on 16-byte boundaries, as its copies to LDS need them (no GPU)."""

import pytest

import paper_2510_08726_amd as pa
from test_train_refusals import at, fwd, lib     # noqa: F401


@pytest.mark.parametrize("n,name", enumerate(("q", "k", "v", "o"), 1))
@pytest.mark.parametrize("off", [2, 4, 8, 14])
def test_tensors_that_are_not_aligned_are_refused(lib, n, name, off):     # noqa: F811
    assert fwd(lib, **{name: at(n, off)}) == pa.ATTN_ERR_SHAPE
