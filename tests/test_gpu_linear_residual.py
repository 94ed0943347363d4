"""Residuals whose rows are aligned but end inside a 16-byte piece: views of a
wider buffer, and one row for all.  The tiled kernels load whole pieces of these
rows at once; the last column of the last row is then the last half of a 32-bit
word that the operand holds half of."""
import pytest
import torch

import scaled_ref as R
from helpers import say
from paper_2009_13108_amd import niti
from test_gpu_linear import ACTS, BF16, F16, F32, codes, floats, forward64, row_scales

pytestmark = pytest.mark.gpu

# rows, odd columns, sum: two tile sizes with more and with less than one tile a CU, and operands at odd addresses
SIZES = [(1000, 1501, 96), (1000, 1501, 95), (2000, 1501, 512), (3001, 2501, 64), (4001, 4001, 128)]


def residual(kind, m, n, dtype):
    """A residual of m x n, and the buffer around it, whose other elements are not numbers."""
    wide = -(-n // 8) * 8 + 8
    if kind == "view":
        buf = torch.full((m, wide), float("nan"), dtype=dtype, device="cuda")
        view = buf[:, :n]
    elif kind == "row":
        buf = torch.full((wide,), float("nan"), dtype=dtype, device="cuda")
        view = buf[:n].expand(m, n)
    else:   # rows whose stride is the width, rounded up: the last row ends the buffer
        ld = -(-n // 8) * 8
        buf = torch.full(((m - 1) * ld + n,), float("nan"), dtype=dtype, device="cuda")
        view = buf.as_strided((m, n), (ld, 1))
    if kind == "row":
        buf[:n] = floats(n, seed=5, dtype=dtype)
    else:
        view.copy_(floats(m, n, seed=5, dtype=dtype))
    return view


@pytest.mark.parametrize("kind", ["view", "row", "end"])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_ragged_residual(m, n, k, dtype, kind):
    say("ragged residual", m, n, k, dtype, kind)
    a, b = codes(m, k, 1), codes(n, k, 2)
    s_a, s_b = row_scales(m, k, 3) * 4, row_scales(n, 1, 4) * 18
    res = residual(kind, m, n, dtype)
    out, intact = R.guarded(m, n, dtype)
    ws = niti.new_workspace(niti.workspace_bytes(niti.OP_LINEAR_FWD, None, m, n, k))
    niti.linear_fwd(a, b, out, s_a, s_b, act=ACTS["relu"], res=res, ws=ws)
    _, _, want, bound = forward64(a, b, s_a, s_b, None, "relu", res)
    R.close(out, want, bound, dtype, "out")
    intact()
    # the edges: the last rows of tiles and the last column, where the products leave the residual as it is
    niti.linear_fwd(torch.zeros_like(a), b, out, s_a, s_b, act=ACTS["relu"], res=res, ws=ws)
    assert torch.equal(out[:, -1], res[:, -1]) and torch.equal(out[-1], res[-1])
