"""The gradient from lse where lse is large: shares of a row are never above 1 by more than lse's rounding."""
import numpy as np
import pytest
import torch

import logits_ref as L
import scaled_ref as R
from paper_2009_13108_amd import niti
from test_gpu_logits import BF16, F16, F32, logits, teacher_of

pytestmark = pytest.mark.gpu


def both(x, tv, ti, scale, dloss):
    m, v = x.shape
    ws = niti.new_workspace(niti.workspace_bytes(niti.OP_DISTILL_FWD, None, m, v))
    loss, lse = torch.empty(m, device="cuda"), torch.empty(m, device="cuda")
    niti.distill_fwd(x, tv, ti, loss, lse=lse, scale=scale, ws=ws)
    dx, intact = R.guarded(m, v, x.dtype, pad=1)
    niti.distill_bwd(x, tv, ti, lse, dloss, dx, scale=scale)
    intact()
    return lse, dx


@pytest.mark.parametrize("scale", [1.0, 0.7, 0.3, 1 / 0.7])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("v", [6, 300, 3000, 140000])
def test_rows_of_the_lowest_value(v, dtype, scale):
    x = logits(4, v, dtype, 41)
    k = min(5, v)
    tv, ti = teacher_of(x, k, 42, F32)
    x[0] = torch.finfo(dtype).min
    x[1, : v - 2] = torch.finfo(dtype).min
    x[2] = torch.finfo(dtype).max
    # (g q, q up to 1 and a share's rounding, less g p; p up to 1)
    for dloss in (torch.tensor([1.0, 0.5, 0.25, 2.0], device="cuda"), torch.tensor([0.0, 0.5, 0.0, 2.0], device="cuda")):
        _, dx = both(x, tv, ti, scale, dloss)
        g = (dloss * scale).double()[:, None]
        assert (dx.double().abs() <= g * (1 + 2.0 ** -6)).all()      # finite among it
        assert (dx[dloss == 0] == 0).all()


@pytest.mark.parametrize("offset", [0.0, 1000.0, -30000.0])
@pytest.mark.parametrize("m,v", [(3, 1), (3, 7), (4, 500), (3, 9000), (2, 140000)])
def test_logits_with_an_offset(m, v, offset):
    """The formula's values from the lse that is given, whatever its rounding: for one column of logits that is all there is."""
    x = logits(m, v, F32, 43) + offset
    k = min(9, v)
    tv, ti = teacher_of(x, k, 44, F32)
    dloss = torch.rand(m, generator=torch.Generator().manual_seed(45)).cuda() + 0.1
    scale = float(np.float32(1 / 0.7))
    lse, dx = both(x, tv, ti, scale, dloss)
    want, off = L.grad64(L.Rows(x, scale), L.Teacher(tv, ti, v, scale), dloss, lse)
    R.close(dx, want, off, what="dx")


def test_not_finite_rows_stay_so():
    x = logits(3, 700, F32, 46)
    tv, ti = teacher_of(x, 4, 47, F32)
    x[0, 5] = float("nan")
    x[1, 6] = float("inf")
    lse, dx = both(x, tv, ti, 0.7, torch.ones(3, device="cuda"))
    assert torch.isnan(lse[:2]).all() and torch.isnan(dx[:2]).all() and torch.isfinite(dx[2]).all()
