"""The gradient in the loss's call where rows are split over workgroups: as close to 64 bits as that of
whole rows, however large the logits are."""
import numpy as np
import pytest
import torch

import logits_ref as L
import scaled_ref as R
from helpers import say
from paper_2009_13108_amd import niti
from test_gpu_logits import BF16, F16, F32, logits, teacher_of

pytestmark = pytest.mark.gpu


def fused(x, tv, ti, scale, dloss, keep=True):
    m, v = x.shape
    ws = niti.new_workspace(niti.workspace_bytes(niti.OP_DISTILL_FWD, None, m, v))
    ws.random_(0, 256)
    loss, lse = torch.full((m,), 7.0, device="cuda"), torch.full((m,), 7.0, device="cuda")
    dx, intact = R.guarded(m, v, x.dtype, pad=1)
    niti.distill_fwd(x, tv, ti, loss, lse=lse if keep else None, dlogits=dx, dloss=dloss, scale=scale, ws=ws)
    intact()
    return dx


def check(x, tv, ti, scale, dloss, base_off=0.0):
    scale = float(np.float32(scale))
    rows, teach = L.Rows(x, scale), L.Teacher(tv, ti, x.shape[1], scale)
    want, off = L.grad64(rows, teach, dloss)
    # joining the parts: a difference of maxima, its product and power (2 U32 for each part's own share of 3 |u|, which grad64
    # has), their product, the power that frees the sum of the base's rounding, a quotient and two products: 10 U32 of q
    off = off + 10 * R.U32 * (dloss.double().cpu().abs() * scale).view(-1, 1) * rows.q
    for keep in (True, False):
        R.close(fused(x, tv, ti, scale, dloss, keep), want, off, x.dtype, "dx")
    return want


@pytest.mark.parametrize("offset", [0.0, 1000.0, -30000.0])
@pytest.mark.parametrize("m,v,dtype", [(3, 60000, F32), (3, 65536, F32), (3, 65537, F32), (2, 131075, F32), (70, 66000, F32), (1, 800001, F32),
                                       (3, 70000, BF16), (2, 131075, F16), (66, 131080, BF16)])
def test_gradient_of_split_rows(m, v, dtype, offset):
    say("split distillation", m, v, dtype, offset)
    x = logits(m, v, F32, 31) + offset
    x = x.to(dtype)
    tv, ti = teacher_of(x, 20, 32, F32)
    dloss = torch.rand(m, generator=torch.Generator().manual_seed(33)).cuda() + 0.1
    check(x, tv, ti, 1 / 0.7, dloss)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("v", [3000, 40000, 65537, 140000])
def test_rows_of_the_lowest_value(v, dtype):
    """A row masked with the type's lowest value throughout: the same share for each, the same as in a whole row."""
    x = logits(4, v, dtype, 34)
    tv, ti = teacher_of(x, 5, 35, F32)
    x[0] = torch.finfo(dtype).min
    x[1] = torch.finfo(dtype).min
    x[1, 5:9] = torch.finfo(dtype).min / 2
    x[2] = torch.finfo(dtype).max
    dloss = torch.tensor([1.0, 0.5, 0.25, 2.0], device="cuda")
    want = check(x, tv, ti, 0.7, dloss)
    assert torch.isfinite(want).all()
    padded = fused(x, tv, ti, 0.7, dloss * torch.tensor([0.0, 1.0, 1.0, 1.0], device="cuda"))
    assert (padded[0] == 0).all()
