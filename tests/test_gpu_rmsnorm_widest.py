"""The widest rows that the norms take: those of no multiple of 8 whose chunks, begun at a multiple of 8 of the matrix, are
one more than 1024 lanes hold, and the widths beside them."""

import pytest

import test_gpu_rmsnorm_add as few
import test_gpu_rmsnorm_turns as many

pytestmark = pytest.mark.gpu

WIDTHS = [32760, 32761, 32762, 32763, 32764, 32765, 32766, 32767]


@pytest.mark.parametrize("M", WIDTHS)
@pytest.mark.parametrize("types", few.TYPES)
def test_against_64_bits(M, types):
    few.test_norm(3, M, types)
    few.test_norm_gradients(3, M, types)


@pytest.mark.parametrize("M", WIDTHS)
@pytest.mark.parametrize("code", ["e4m3", "int8"])
def test_in_8_bits(M, code):
    for types in few.TYPES:
        few.test_norm_in_8_bits(2, M, code, types)


@pytest.mark.parametrize("M", [32761, 32762, 32767])
@pytest.mark.parametrize("types", many.TYPES)
def test_rows_in_turn(M, types):
    """(256 workgroups of a row each; to 8 bits as many.)"""
    many.test_rows_in_turn(515, M, types)
    many.test_gradients_of_rows_in_turn(515, M, types)
