"""Choices of the row operators, seen through the workspace sizes (which need no GPU)."""
import pytest

from paper_2009_13108_amd import niti


@pytest.mark.parametrize("d, few", [(64, 16), (512, 16), (1000, 16), (1024, 16), (1025, 3), (1111, 3), (4096, 3), (4097, 2), (9216, 2), (40000, 2)])
def test_few_rows_of_the_norm_go_by_one_workgroup(d, few):
    """Up to so many rows one launch beats two (4 rows of 4096: 6.4 us against 6.0): one partial row, which is dgain."""
    def parts(m):
        return niti.workspace_bytes(niti.OP_RMSNORM_BWD, None, m, d) // (-(-d * 4 // 256) * 256)
    assert parts(1) == 1 and parts(few) == 1
    assert parts(few + 1) > 1
