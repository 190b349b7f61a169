"""Workspace of the weights' gradient with a kept x, on the CPU: no less than that of the gradient itself, also where x has no columns."""
import pytest

from paper_2207_04606_amd import moe


@pytest.mark.parametrize("d_in", [0, 1, 40, 1024])
@pytest.mark.parametrize("rows,experts,d_z", [(9000, 1, 64), (12000, 3, 24), (300, 1, 64), (9000, 1, 0)])
def test_no_less_than_without(rows, experts, d_z, d_in):
    lib = moe._library()
    plain = lib.sptir_moe_product_dw_workspace(rows, experts, d_in, d_z)
    for kind in moe.TYPES.values():
        packed = lib.sptir_moe_product_dw_packed_workspace(kind, rows, rows, experts, d_in, d_z)
        assert packed >= plain
        assert d_in > 0 or packed == plain
    assert plain > 0 or (rows, d_z) != (9000, 64)
