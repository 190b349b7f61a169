"""Which kernel takes a product of 8-bit integers or a gradient through a z kept in 8 bits (csrc/moe_choice.h): the sizes of test_gpu_moe_int8_wide.py and
test_gpu_moe_packed_wide.py take more tiles of 256 x 256 than the card has CUs."""
import pytest

import moe_wide_shapes as wide
from test_moe_choice import choice  # noqa: F401


@pytest.mark.parametrize("T,k,E,d_in,d_out,act,dropped", wide.INT8)
def test_large_tiles_of_8_bit_integers(choice, T, k, E, d_in, d_out, act, dropped):  # noqa: F811
    # (the estimates take 8-bit integers for half as many of 16 bits, whatever the type of y; rows in 16-byte words for all of them)
    few, is_wide, _, _ = choice("forward", T * k, max(E, 1), E > 0, wide.columns(d_out, act), (d_in + 1) // 2, 0, 1, act == "swiglu")
    assert not few and is_wide
    assert d_in % 16 == 0 and d_out % 8 == 0
    assert wide.tiles(T * k * (1 - dropped), wide.columns(d_out, act)) > 256


@pytest.mark.parametrize("T,k,E,d_in,d_z,acts,dropped", wide.DX_KEPT)
def test_large_tiles_through_a_kept_z(choice, T, k, E, d_in, d_z, acts, dropped):  # noqa: F811
    assert choice("dx", T * k, max(E, 1), E > 0, d_in, d_z, 0, 1, 0)[:2] == (0, 1)
    assert d_in % 8 == 0 and d_z % 8 == 0
    assert wide.tiles(T * k * (1 - dropped), d_in) > 256


def test_few_rows_without_inputs(choice):  # noqa: F811
    """Rows and columns of test_gpu_moe_no_inputs.py: the kernel for few rows takes calls without inputs too."""
    assert choice("forward", 20000, 1, 0, 2048, 0, 0, 1, 0)[0] == 1
    assert choice("forward", 500, 1, 0, 24, 0, 0, 1, 0)[0] == 0


def test_few_rows_beside_many(choice):  # noqa: F811
    """The two calls of test_gpu_moe_int8_wide.py whose rows have to be equal take different kernels."""
    assert choice("forward", 16, 1, 0, 7640, 328, 0, 1, 0)[0] == 1
    assert choice("forward", 3700, 1, 0, 7640, 328, 0, 1, 0)[:2] == (0, 1)
