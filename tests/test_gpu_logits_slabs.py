"""Calls on logits of more rows than a launch takes: the rows of every launch have their own operands and
outputs.  And workspaces that were sized for more rows than a call has."""
import pytest
import torch

from helpers import say
from paper_2009_13108_amd import niti
from test_gpu_logits import BF16, F16, F32, logits, some_tokens, teacher_of

pytestmark = pytest.mark.gpu
SLAB = 1 << 21          # workgroups of a launch


def logprobs(x, tok, top, ws):
    m = x.shape[0]
    out = {k: torch.full((m,), 7.0, device="cuda") for k in ("logp", "lse", "entropy")}
    out["top_logp"], out["top_idx"] = torch.full((m, top), 7.0, device="cuda"), torch.full((m, top), 7, dtype=torch.int32, device="cuda")
    niti.token_logprobs(x, tokens=tok, scale=0.7, ws=ws, **out)
    return out


def distill(x, tv, ti, dloss, ws, dx=None):
    m = x.shape[0]
    loss, lse = torch.full((m,), 7.0, device="cuda"), torch.full((m,), 7.0, device="cuda")
    dx = torch.full_like(x, 7.0) if dx is None else dx
    niti.distill_fwd(x, tv, ti, loss, lse=lse, dlogits=dx, dloss=dloss, scale=0.7, ws=ws)
    return loss, lse, dx


def some_rows(m, edges):
    """The first rows, those about each edge, the last."""
    return sorted({r for e in (2, *edges, m) for r in range(max(0, e - 3), min(m, e + 3))})


@pytest.mark.parametrize("v", [6, 9])
def test_more_rows_than_a_launch(v):
    m = SLAB + 3
    say("logits", m, v)
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(m, v, generator=g, device="cuda")
    tok = torch.randint(0, v, (m,), generator=g, device="cuda").to(torch.int32)
    tv, ti = torch.randn(m, 3, generator=g, device="cuda"), torch.randint(0, v, (m, 3), generator=g, device="cuda").to(torch.int32)
    dloss = torch.rand(m, generator=g, device="cuda")
    at = torch.tensor(some_rows(m, [SLAB]), device="cuda")
    # (a row's results are its own: no other row of a call comes into them)
    every, few = logprobs(x, tok, 4, None), logprobs(x[at], tok[at], 4, None)
    for k in few:
        assert torch.equal(every[k][at], few[k]), k
    every, few = distill(x, tv, ti, dloss, None), distill(x[at], tv[at], ti[at], dloss[at], None)
    assert all(torch.equal(a[at], b) for a, b in zip(every, few))
    dx = torch.full_like(x, 7.0)
    niti.distill_bwd(x, tv, ti, every[1], dloss, dx, scale=0.7)
    part = torch.full_like(x[at], 7.0)
    niti.distill_bwd(x[at], tv[at], ti[at], few[1], dloss[at], part, scale=0.7)
    assert torch.equal(dx[at], part)


def test_more_split_rows_than_a_launch():
    """Rows of the same logits (stride 0) with tokens, lists and weights of their own."""
    v = 32769
    m = SLAB // 3 + 5
    say("split logits", m, v)
    x = logits(1, v, BF16, 2).expand(m, v)
    tok = some_tokens(m, v, 3)
    ws = niti.new_workspace(niti.workspace_bytes(niti.OP_TOKEN_LOGPROBS, None, m, v, 4))
    at = torch.tensor(some_rows(m, [SLAB // 3]), device="cuda")
    every = logprobs(x, tok, 4, ws)
    few = logprobs(x[:300], torch.cat([tok[at], tok[:300 - len(at)]]), 4, ws)          # (more than 256: in the same parts)
    for k in few:
        assert torch.equal(every[k][at], few[k][:len(at)]), k
    assert torch.equal(every["lse"], every["lse"][:1].expand(m)) and (every["top_idx"] == every["top_idx"][:1]).all()
    del every, few, ws

    v, parts = 131073, 17
    m = SLAB // parts + 3
    if torch.cuda.mem_get_info()[0] < 80 << 30:
        pytest.skip("the gradient takes 32 GB")
    say("split distillation", m, v)
    x = logits(1, v, BF16, 4).expand(m, v)
    g = torch.Generator(device="cuda").manual_seed(5)
    tv, ti = torch.randn(m, 3, generator=g, device="cuda"), torch.randint(0, v, (m, 3), generator=g, device="cuda").to(torch.int32)
    dloss = torch.rand(m, generator=g, device="cuda")
    dx = torch.empty(m, v, dtype=BF16, device="cuda")
    ws = niti.new_workspace(niti.workspace_bytes(niti.OP_DISTILL_FWD, None, m, v))
    loss, lse, _ = distill(x, tv, ti, dloss, ws, dx)
    at = torch.tensor(some_rows(m, [SLAB // 33, SLAB // parts]), device="cuda")          # the gradient has 33 parts a row
    few = distill(x[:len(at)], tv[at], ti[at], dloss[at], ws, torch.empty(len(at), v, dtype=BF16, device="cuda"))
    assert torch.equal(loss[at], few[0]) and torch.equal(lse[at], few[1]) and torch.equal(dx[at], few[2])


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("v", [20001, 40001, 100003, 140000])
def test_workspace_of_many_rows(v, dtype):
    """A batch's workspace serves smaller batches."""
    many, top = 300, 20
    x, tok = logits(many, v, dtype, 6), some_tokens(many, v, 7)
    tv, ti = teacher_of(x, 9, 8, F32)
    dloss = torch.rand(many, generator=torch.Generator().manual_seed(9)).cuda()
    ws = niti.new_workspace(max(niti.workspace_bytes(niti.OP_TOKEN_LOGPROBS, None, many, v, top), niti.workspace_bytes(niti.OP_DISTILL_FWD, None, many, v)))
    for m in (300, 257, 97, 49, 48, 1):
        own = niti.new_workspace(max(niti.workspace_bytes(niti.OP_TOKEN_LOGPROBS, None, m, v, top), niti.workspace_bytes(niti.OP_DISTILL_FWD, None, m, v)))
        ws.random_(0, 256)
        a, b = logprobs(x[:m], tok[:m], top, ws), logprobs(x[:m], tok[:m], top, own)
        assert all(torch.equal(a[k], b[k]) for k in a), m
        ws.random_(0, 256)
        a, b = distill(x[:m], tv[:m], ti[:m], dloss[:m], ws), distill(x[:m], tv[:m], ti[:m], dloss[:m], own)
        assert all(torch.equal(s, t) for s, t in zip(a, b)), m
