"""The table's gradient in types that differ from the errors', and of tables with more than 2^24 rows, whose
tokens take four passes to sort."""
import pytest
import torch

import scaled_ref as R
import test_gpu_embedding as E
from helpers import say
from paper_2009_13108_amd import niti

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,grad", [(E.F16, E.F32), (E.F32, E.F16), (E.BF16, E.F16), (E.F16, E.BF16)])
@pytest.mark.parametrize("m,v,d,kind", E.SHAPES)
def test_other_types(m, v, d, kind, dtype, grad):
    E.test_backward(m, v, d, kind, dtype, grad)


@pytest.mark.parametrize("m", [700, 9000, 40000])
def test_many_rows(m):
    """The highest tokens, ones that differ in each of their bytes, some often, some outside the table."""
    v, d, alpha = (1 << 24) + 70000, 2, float(torch.tensor(1.7))
    say("embedding_bwd", m, v, d)
    g = torch.Generator().manual_seed(7)
    tok = torch.randint(0, v, (m,), generator=g)
    tok[::3] = torch.randint(0, 256, (len(tok[::3]),), generator=g) << 16
    tok[1::7] = v - 1 - torch.randint(0, 5, (len(tok[1::7]),), generator=g)
    tok[2::11] = v + torch.randint(0, 3, (len(tok[2::11]),), generator=g)
    dy = E.floats(m, d, seed=8)
    ws = niti.new_workspace(niti.workspace_bytes(niti.OP_EMBEDDING_BWD, None, m, v, d))
    ws.random_(0, 256)
    out = torch.full((v, d), 7.0, device="cuda")
    niti.embedding_bwd(dy, tok.to(torch.int32).cuda(), out, ws, alpha=alpha)
    inside = tok < v
    seen, at, n = torch.unique(tok[inside], return_inverse=True, return_counts=True)
    rows = dy.double().cpu()[inside]
    zero = torch.zeros(len(seen), d, dtype=torch.float64)
    want, mags = alpha * zero.index_add(0, at, rows), zero.index_add(0, at, rows.abs())
    bound = 1.01 * R.U32 * (alpha * n[:, None] * mags + 2 * want.abs())
    where = seen.cuda()
    R.close(out[where], want, bound, E.F32, "dtable")
    out[where] = 0
    assert not out.any()
    out.fill_(0.5)
    niti.embedding_bwd(dy, tok.to(torch.int32).cuda(), out, ws, alpha=alpha, accumulate=True)
    R.close(out[where], want + 0.5, bound + 1.01 * R.U32 * (want + 0.5).abs(), E.F32, "accumulated")
    out[where] = 0.5
    assert (out == 0.5).all()
