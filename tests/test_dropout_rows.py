"""How the rows of dropout's bias gradient are shared out over blocks, each of which leaves a row of float32 sums in the workspace.  No GPU needed."""
import pytest

from paper_2411_15871_amd import dhelix as dh


@pytest.mark.parametrize("T", [2 ** 31 - 1, 2 ** 31 - 10, 2 ** 31 - 2000, 2 ** 30])
def test_rows_up_to_the_last_of_32_bits(T):
    """2048 blocks of rows for one of columns, also where the rows' count rounded up passes 32 bits."""
    assert dh.dh_dropout_add_bwd_ws_bytes(T, 8) == 2048 * 8 * 4
