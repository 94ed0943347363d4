"""Embedding lookup and the table's gradient against 64-bit forms.

A lookup rounds once (two factors: twice).  A sum of n terms in any order is off by at most
(n - 1) U32 of the sum of their magnitudes, to first order (n U32 here), its product with alpha
and the addition to what is there by one rounding each."""
import numpy as np
import pytest
import torch

import scaled_ref as R
from helpers import say
from paper_2009_13108_amd import niti

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def floats(*shape, seed, dtype=F32, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(dtype).cuda()


def tokens_of(m, v, seed, kind="zipf"):
    g = torch.Generator().manual_seed(seed)
    if kind == "zipf":
        t = (torch.exp(torch.rand(m, generator=g) * np.log(v + 1.0)) - 1).long().clamp(max=v - 1)
    elif kind == "one":
        t = torch.full((m,), v - 1)
    elif kind == "runs":      # a few tokens, each many times
        t = torch.randint(0, min(v, 5), (m,), generator=g) * (v // 5 if v >= 5 else 1)
    else:                     # "holes": some outside the table
        t = torch.randint(-2, v + 2, (m,), generator=g)
    return t.to(torch.int32).cuda()


F = float(np.float32(1.7))


@pytest.mark.parametrize("table", [F32, BF16, F16, torch.int8])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("m,v,d", [(1, 1, 1), (1, 7, 3), (5, 3, 7), (8, 1000, 8), (33, 50, 65), (7, 300, 1111), (300, 40, 4096), (2, 9, 8200)])
def test_forward(m, v, d, table, dtype):
    say("embedding_fwd", m, v, d, table, dtype)
    tok = tokens_of(m, v, 1, "holes" if m > 4 else "zipf")
    scale = None
    if table is torch.int8:
        t = torch.randint(-127, 128, (v, d + 3), generator=torch.Generator().manual_seed(2), dtype=torch.int8).cuda()[:, :d]
        scale = floats(v, seed=3).abs() + 0.1
    else:
        t = floats(v, d + 5, seed=2, dtype=table)[:, :d]
    out, intact = R.guarded(m, d, dtype, pad=3)
    niti.embedding_fwd(t, tok, out, table_scale=scale, alpha=1.7)
    at = tok.long().cpu()
    inside = (at >= 0) & (at < v)
    rows = t.double().cpu()[at.clamp(0, v - 1)] * F
    if scale is not None:
        rows = rows * scale.double().cpu()[at.clamp(0, v - 1)][:, None]
    rows = torch.where(inside[:, None], rows, torch.zeros_like(rows))
    R.close(out, rows, 2.01 * R.U32 * rows.abs(), dtype, "out")
    assert (out.cpu()[~inside] == 0).all()
    intact()


def test_forward_keeps_values():
    """alpha 1: the table's own values, infinities and NaNs among them; rows that no token names are not read into others."""
    t = floats(6, 40, seed=1)
    t[1, 3], t[2, 4], t[3] = float("inf"), float("nan"), float("nan")
    tok = torch.tensor([5, 1, 2, 0, -1, 6, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device="cuda")
    out = torch.empty(8, 40, device="cuda")
    niti.embedding_fwd(t, tok, out)
    assert torch.equal(out[0], t[5]) and torch.equal(out[1], t[1]) and torch.equal(out[3], t[0])
    assert torch.isnan(out[2, 4]) and torch.isfinite(out[2, 5:]).all() and (out[4:] == 0).all()
    niti.embedding_fwd(t, tok[:0], out[:0])


def backward64(dy, tok, v, alpha, old=None):
    at = tok.long().cpu()
    inside = (at >= 0) & (at < v)
    at, dy = at[inside], dy.double().cpu()[inside]
    zero = torch.zeros(v, dy.shape[1], dtype=torch.float64)
    sums, mags = zero.index_add(0, at, dy), zero.index_add(0, at, dy.abs())
    n = torch.zeros(v, dtype=torch.float64).index_add(0, at, torch.ones(len(at), dtype=torch.float64))
    want = alpha * sums + (old.double().cpu() if old is not None else 0)
    return want, 1.01 * R.U32 * (abs(alpha) * n[:, None] * mags + 2 * want.abs()), n


SHAPES = [(1, 1, 1, "one"), (1, 50, 9, "zipf"), (15, 20, 3, "runs"), (16, 4, 8, "one"), (17, 300, 64, "holes"), (100, 33, 1111, "zipf"),
          (257, 70000, 16, "zipf"), (1000, 257, 200, "holes"), (1025, 256, 72, "runs"), (1024, 255, 40, "zipf"), (3000, 9000, 2056, "zipf"),
          (5000, 2, 2049, "one"), (4096, 500, 4100, "runs"), (16384, 300, 24, "zipf"), (16385, 70000, 20, "zipf"), (40000, 1000, 33, "holes"),
          (70001, 11, 8, "runs"), (33000, 66000, 7, "one")]


@pytest.mark.parametrize("dtype,grad", [(F32, F32), (BF16, BF16), (BF16, F32), (F16, F16), (F32, BF16)])
@pytest.mark.parametrize("m,v,d,kind", SHAPES)
def test_backward(m, v, d, kind, dtype, grad):
    say("embedding_bwd", m, v, d, kind, dtype, grad)
    tok = tokens_of(m, v, 4, kind)
    dy = floats(m, d + 1, seed=5, dtype=dtype)[:, :d]
    ws = niti.new_workspace(niti.workspace_bytes(niti.OP_EMBEDDING_BWD, None, m, v, d))
    ws.random_(0, 256)
    out, intact = R.guarded(v, d, grad, pad=1)
    niti.embedding_bwd(dy, tok, out, ws, alpha=1.7)
    want, bound, n = backward64(dy, tok, v, F)
    R.close(out, want, bound, grad, "dtable")
    assert (out.cpu()[n == 0] == 0).all()
    intact()
    first = out.clone()
    ws.random_(0, 256)
    niti.embedding_bwd(dy, tok, out, ws, alpha=1.7)
    assert torch.equal(out, first)                 # the order of the sums is fixed
    old = floats(v, d, seed=6, dtype=grad)
    old[n.cuda() == 0] = float("nan")              # rows of no token are left as they are, whatever they hold
    out.copy_(old)
    niti.embedding_bwd(dy, tok, out, ws, alpha=1.7, accumulate=True)
    want, bound, _ = backward64(dy, tok, v, F, old)
    R.close(out, want, bound, grad, "accumulated")
    intact()


def test_backward_is_the_lookups_gradient():
    """<dy, lookup(table + e t) - lookup(table - e t)> / 2e = <dtable, t>, in 64 bits on the host for the lookup."""
    m, v, d = 200, 30, 50
    tok, dy = tokens_of(m, v, 1, "holes"), floats(200, 50, seed=2)
    out = torch.empty(v, d, device="cuda")
    niti.embedding_bwd(dy, tok, out, niti.new_workspace(niti.workspace_bytes(niti.OP_EMBEDDING_BWD, None, m, v, d)), alpha=0.5)
    at = tok.long().cpu()
    inside = ((at >= 0) & (at < v)).double()[:, None]
    t = torch.randn(v, d, dtype=torch.float64, generator=torch.Generator().manual_seed(3))
    want = (0.5 * t[at.clamp(0, v - 1)] * inside * dy.double().cpu()).sum()
    got = (out.double().cpu() * t).sum()
    _, bound, _ = backward64(dy, tok, v, 0.5)
    assert abs(float(got - want)) <= float((bound * t.abs()).sum())


def test_backward_edges():
    out = torch.full((5, 12), 7.0, device="cuda")
    dy, tok = torch.ones(0, 12, device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda")
    niti.embedding_bwd(dy, tok, out, None, accumulate=True)
    assert (out == 7).all()
    niti.embedding_bwd(dy, tok, out, None)
    assert (out == 0).all()
    # one row for all tokens (stride 0), none of them in the table, a value that is not finite in one token's rows only
    ws = niti.new_workspace(niti.workspace_bytes(niti.OP_EMBEDDING_BWD, None, 40, 5, 12))
    row = floats(1, 12, seed=1)
    tok = torch.arange(40, dtype=torch.int32, device="cuda") % 4
    niti.embedding_bwd(row.expand(40, 12), tok, out, ws)
    R.close(out[:4], 10 * row.expand(4, 12).double(), 10 * R.U32 * 10 * row.abs().double().cpu(), what="stride 0")
    assert (out[4] == 0).all()
    niti.embedding_bwd(row.expand(40, 12), tok - 100, out, ws)
    assert (out == 0).all()
    dy = floats(40, 12, seed=2)
    dy[6, 3] = float("inf")
    niti.embedding_bwd(dy, tok, out, ws)
    assert out[2, 3] == float("inf") and int(torch.isfinite(out).sum()) == 59


def test_past_32_bit_offsets():
    """Table, gradient and errors beyond 2^31 bytes: rows far apart."""
    v, d, ld = 600, 40, (1 << 20) - 8
    big = torch.empty(v * ld, device="cuda")          # 2.5 GB
    wide = big.as_strided((v, d), (ld, 1))
    table = floats(v, d, seed=1)
    wide.copy_(table)
    tok = torch.arange(v, dtype=torch.int32, device="cuda").flip(0).contiguous()
    out = torch.empty(v, d, device="cuda")
    niti.embedding_fwd(wide, tok, out)
    assert torch.equal(out, table.flip(0))
    ws = niti.new_workspace(niti.workspace_bytes(niti.OP_EMBEDDING_BWD, None, v, v, d))
    niti.embedding_bwd(wide, tok, out, ws)
    assert torch.equal(out, table.flip(0))
    niti.embedding_bwd(table, tok, wide, ws)
    assert torch.equal(wide.contiguous(), table.flip(0))


def test_stream_and_graph():
    m, v, d = 20000, 500, 96
    tok, dy, out = tokens_of(m, v, 1), floats(m, d, seed=2, dtype=BF16), torch.empty(v, d, device="cuda")
    ws = niti.new_workspace(niti.workspace_bytes(niti.OP_EMBEDDING_BWD, None, m, v, d))
    table, x = floats(v, d, seed=3), torch.empty(m, d, dtype=BF16, device="cuda")

    def step():
        niti.embedding_fwd(table, tok, x, alpha=2.0)
        niti.embedding_bwd(dy, tok, out, ws)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in range(3):
        tok.copy_(tokens_of(m, v, 10 + seed))
        dy.copy_(floats(m, d, seed=20 + seed, dtype=BF16))
        step()
        want = [x.clone(), out.clone()]
        x.zero_(), out.fill_(5), ws.random_(0, 256)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(x, want[0]) and torch.equal(out, want[1])


def test_refusals():
    table, tok, out = torch.ones(5, 8, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda"), torch.empty(3, 8, device="cuda")
    with pytest.raises(TypeError):
        niti.embedding_fwd(table, tok.long(), out)
    with pytest.raises(ValueError):
        niti.embedding_fwd(table, tok, out[:2])
    with pytest.raises(ValueError):
        niti.embedding_fwd(table, tok, out, table_scale=torch.ones(5, device="cuda"))
    with pytest.raises(ValueError):
        niti.embedding_fwd(table.to(torch.int8), tok, out)
    with pytest.raises(TypeError):
        niti.embedding_fwd(table.double(), tok, out)
    with pytest.raises(niti.NitiError):
        niti.embedding_fwd(table, tok, out, alpha=float("inf"))
    with pytest.raises(niti.NitiError):
        niti.embedding_bwd(out, tok, table, None)
    with pytest.raises(niti.NitiError):
        niti.embedding_bwd(out, tok, table, niti.new_workspace(64))
    with pytest.raises(ValueError):
        niti.embedding_bwd(out, tok[:2], table, niti.new_workspace(1 << 16))
    with pytest.raises(TypeError):
        niti.embedding_bwd(out, None, table, niti.new_workspace(1 << 16))
