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


def test_sizes_that_no_call_takes_need_no_workspace():
    """As niti_linear_fwd's: 0, and no product of sizes that leaves 64 bits."""
    big = 1 << 61
    for op, sizes in ((niti.OP_RMSNORM_BWD, [(1 << 31, 8, 0), (8, 1 << 22, 0), (8, big, 0), (big, 8, 0)]),
                      (niti.OP_LINEAR_FWD, [(1 << 31, 8, 8), (8, 1 << 22, 8), (8, 8, 1 << 17), (big, big, big)]),
                      (niti.OP_LINEAR_BWD, [(1 << 17, 8, 8), (8, 1 << 17, 8), (8, 8, 1 << 22), (big, 8, 8), (8, 8, big), (big, big, big)])):
        for m, n, k in sizes:
            assert niti.workspace_bytes(op, None, m, n, k) == 0, (op, m, n, k)
    assert niti.workspace_bytes(niti.OP_LINEAR_BWD, None, (1 << 17) - 1, 8, 8) > 0
    assert niti.workspace_bytes(niti.OP_LINEAR_BWD, None, 8, 8, (1 << 22) - 1) > 0
    assert niti.workspace_bytes(niti.OP_RMSNORM_BWD, None, 8, (1 << 22) - 1) > 0
