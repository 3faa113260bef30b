"""More refusals of the block ends' entry points, on the host: no GPU is touched."""
import pytest

from tests.test_block_ops_abi import DIM, INVALID, NEED, ROWS, B, at, branch, branch_desc  # noqa: F401


@pytest.mark.parametrize("per", [ROWS, ROWS + 1, 1 << 40, (1 << 63) - ROWS, (1 << 63) - 1])
def test_a_gate_of_one_row_is_kept_apart_from_what_is_written(B, per):  # noqa: F811
    """However many rows it is for: the gate's size does not overflow."""
    L, d = B.lib(), branch_desc(B, rows_per_gate=per)
    for shift in (0, 4 * DIM - 4):
        assert L.asi_branch_forward(d, branch(B, x=at(2) + shift), None) == INVALID
        assert L.asi_branch_backward(d, branch(B, dnext_weight=at(2) + shift), 0, at(60), NEED, None) == INVALID
