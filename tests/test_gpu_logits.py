"""Log probabilities, entropy and top alternatives of logits, and distillation from a teacher's
top logits, against 64-bit forms (tests/logits_ref.py has the bounds)."""
import numpy as np
import pytest
import torch

import logits_ref as L
import scaled_ref as R
from helpers import say
from paper_2009_13108_amd import niti

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
NINF = float("-inf")


def logits(m, v, dtype, seed, spread=3.0, pad=0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(m, v + pad, generator=g) * spread).to(dtype).cuda()[:, :v]


def some_tokens(m, v, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randint(0, v, (m,), generator=g).to(torch.int32).cuda()


def f32(x):
    return float(np.float32(x))


def run_logprobs(x, tok, top, scale):
    m, v = x.shape
    ws = niti.new_workspace(niti.workspace_bytes(niti.OP_TOKEN_LOGPROBS, None, m, v, top))
    ws.random_(0, 256)
    out = {k: torch.full((m,), 7.0, device="cuda") for k in ("logp", "lse", "entropy")}
    if top:
        out["top_logp"], out["top_idx"] = torch.full((m, top), 7.0, device="cuda"), torch.full((m, top), 7, dtype=torch.int32, device="cuda")
    niti.token_logprobs(x, tokens=tok, scale=scale, ws=ws, **out)
    return out


def check_logprobs(x, tok, top, scale):
    out = run_logprobs(x, tok, top, scale)
    rows = L.Rows(x, f32(scale))
    R.close(out["lse"], rows.lse, rows.lse_off, what="lse")
    R.close(out["entropy"], rows.entropy, rows.entropy_off, what="entropy")
    inside = ((tok >= 0) & (tok < x.shape[1])).cpu()
    lp, off = rows.logp(tok.long().cpu().clamp(0, x.shape[1] - 1)[:, None])
    R.close(out["logp"], torch.where(inside, lp[:, 0], torch.zeros_like(lp[:, 0])), off[:, 0], what="logp")
    if top:
        cols = rows.top(top)
        assert torch.equal(out["top_idx"].long().cpu(), cols), "columns"
        lp, off = rows.logp(cols)
        R.close(out["top_logp"], lp, off, what="top_logp")


# every shape of the kernel and its edges: rows of 512, 2048, 4096, ... columns by a workgroup, and rows in parts
WIDTHS = [(3, 1), (2, 3), (5, 7), (4, 8), (3, 9), (6, 300), (9, 511), (4, 512), (3, 513), (2, 2048), (3, 2051), (2, 4097), (3, 8192),
          (2, 8200), (2, 16385), (3, 32000), (2, 40001), (1, 65536), (2, 65537), (1, 131072), (3, 131075), (1, 200001), (1, 300000), (130, 66000)]


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("m,v", WIDTHS)
def test_logprobs(m, v, dtype):
    say("token_logprobs", m, v, dtype)
    x, tok = logits(m, v, dtype, 1, pad=v % 5), some_tokens(m, v, 2)
    for top, scale in ((0, 1.0), (1, 0.5), (20, 1 / 0.7), (64, 3.0)):
        if top <= v:
            check_logprobs(x, tok, top, scale)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("m,v", [(520, 34000), (513, 17001), (1, 800001), (1, 1200001), (1, 3000001), (70, 90000)])
def test_many_or_very_long_rows(m, v, dtype):
    """Rows in parts of each size, up to the widest rows; and whole rows of the widest kernel."""
    say("logits", m, v, dtype)
    x, tok = logits(m, v, dtype, 1), some_tokens(m, v, 2)
    check_logprobs(x, tok, 20, 0.7)
    if m < 100:
        tv, ti = teacher_of(x, 20, 12, dtype)
        check_distill(x, tv, ti, 0.7, torch.full((m,), 0.25, device="cuda"))


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("m,v", [(5, 1023), (5, 1537), (4, 2560), (4, 2561), (3, 6151), (3, 10000), (3, 12287), (2, 24577), (3, 33281), (300, 40003),
                                 (600, 20001)])
def test_rows_that_end_between_waves(m, v, dtype):
    """A row's end in the middle of a workgroup's columns: waves with fewer pieces than others, with one that is cut, or with none."""
    say("logits", m, v, dtype)
    x, tok = logits(m, v, dtype, 5), some_tokens(m, v, 6)
    for top in (0, 9):
        check_logprobs(x, tok, top, 1.3)
    tv, ti = teacher_of(x, 30, 7, dtype)
    check_distill(x, tv, ti, 1.3, torch.full((m,), 0.5, device="cuda"))
    x[0, : v - 3] = NINF
    x[1, 2:] = NINF
    check_logprobs(x, tok, 9, 1.3)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("v", [40, 700, 5000, 33000, 140000])
def test_equal_logits(v, dtype):
    """Ties go to the lowest column: all equal, few distinct values, rows in order, zeros of both signs."""
    x = torch.stack([torch.full((v,), 2.5), torch.arange(v) % 3 - 1.0, torch.arange(v) * (8.0 / v), -torch.arange(v) * (8.0 / v),
                     torch.where(torch.arange(v) % 2 == 0, 0.0, -0.0), torch.zeros(v)])
    x[5, v - 30:] = 1.0
    x = x.to(dtype).cuda()
    tok = some_tokens(6, v, 3)
    for top in (1, 5, 20, min(64, v)):
        check_logprobs(x, tok, top, 1.0)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("v", [64, 3000, 32000, 140000])
def test_masks(v, dtype):
    """Minus infinity and the type's lowest value as masks; rows that leave fewer than `top`, one, or nothing."""
    x = logits(9, v, dtype, 4)
    x[0, 5:] = NINF
    x[1] = NINF
    x[2, : v - 3] = torch.finfo(dtype).min
    x[3, torch.arange(v) != v // 2] = NINF
    x[4, ::2] = NINF
    x[5] = torch.finfo(dtype).min
    x[6, 0] = torch.finfo(dtype).max
    x[7] = torch.finfo(dtype).max
    x[8, :v // 2] = NINF
    tok = torch.tensor([0, 1, v - 1, v // 2, 0, 3, 0, 9, v - 1], dtype=torch.int32, device="cuda")
    check_logprobs(x, tok, 20, 1.0)
    check_logprobs(x, tok, 64, 0.5)
    tok = torch.tensor([-1, v, -100, 2 ** 31 - 1, -2 ** 31, 3, 0, 9, v - 1], dtype=torch.int32, device="cuda")
    check_logprobs(x, tok, 1, 1.0)


@pytest.mark.parametrize("v", [50, 9000, 140000])
def test_rows_that_are_not_finite(v):
    x = logits(6, v, F32, 5)
    x[1, 7] = float("nan")
    x[2, v - 1] = float("inf")
    x[3] = float("nan")
    x[4, 0], x[4, 1:] = float("nan"), NINF
    tok = some_tokens(6, v, 6)
    out = run_logprobs(x, tok, 20, 1.0)
    for k in ("logp", "lse", "entropy", "top_logp"):
        assert torch.isnan(out[k][1:5]).all(), k
    assert (out["top_idx"][1:5] == -1).all()
    fine = x[[0, 5]].contiguous()
    alone = run_logprobs(fine, tok[[0, 5]].contiguous(), 20, 1.0)
    assert all(torch.equal(out[k][[0, 5]], alone[k]) for k in out)        # no other row is touched


def test_outputs_alone_and_no_rows():
    x, tok = logits(5, 1000, BF16, 7), some_tokens(5, 1000, 8)
    every = run_logprobs(x, tok, 4, 1.0)
    for name in ("lse", "entropy", "top_logp", "top_idx"):
        out = torch.zeros_like(every[name])
        niti.token_logprobs(x, **{name: out})
        assert torch.equal(out, every[name]), name
    out = torch.zeros(5, device="cuda")
    niti.token_logprobs(x, tokens=tok, logp=out)
    assert torch.equal(out, every["logp"])
    niti.token_logprobs(x[:0], lse=out[:0])
    row = x[:1].expand(5, 1000)                                               # stride 0
    niti.token_logprobs(row, lse=out)
    assert (out == every["lse"][0]).all()


# ------------------------------------------------------------------ distillation
def teacher_of(x, k, seed, dtype):
    """The top logits of a teacher near the student, in a buffer of wider rows."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = torch.where(torch.isfinite(x), x.float(), torch.zeros((), device="cuda")) + torch.randn(x.shape, generator=g, device="cuda")
    val, idx = torch.topk(t, k, dim=1)
    wide = torch.zeros(x.shape[0], k + 3, device="cuda", dtype=dtype)
    wide[:, :k] = val.to(dtype)
    return wide[:, :k], idx.to(torch.int32)


def run_distill(x, tv, ti, scale, dloss, in_place=False):
    m, v = x.shape
    ws = niti.new_workspace(niti.workspace_bytes(niti.OP_DISTILL_FWD, None, m, v))
    ws.random_(0, 256)
    loss, lse, alone = (torch.full((m,), 7.0, device="cuda") for _ in range(3))
    dx, intact = R.guarded(m, v, x.dtype, pad=1)
    niti.distill_fwd(x, tv, ti, loss, lse=lse, dlogits=dx, dloss=dloss, scale=scale, ws=ws)
    intact()
    niti.distill_fwd(x, tv, ti, alone, scale=scale, ws=ws)
    assert torch.equal(alone.nan_to_num(nan=-1.0), loss.nan_to_num(nan=-1.0))
    dx2, intact = R.guarded(m, v, x.dtype, pad=2)
    niti.distill_bwd(x, tv, ti, lse, dloss, dx2, scale=scale)
    intact()
    for how in (0, 1):          # over the logits themselves
        y = x.clone()
        if how:
            niti.distill_bwd(y, tv, ti, lse, dloss, y, scale=scale)
        else:
            niti.distill_fwd(y, tv, ti, alone, dlogits=y, dloss=dloss, scale=scale, ws=ws)
        assert torch.equal(y.nan_to_num(nan=3.0), (dx2 if how else dx).nan_to_num(nan=3.0)), how
    return loss, lse, dx, dx2


def check_distill(x, tv, ti, scale, dloss):
    loss, lse, dx, dx2 = run_distill(x, tv, ti, scale, dloss)
    rows, teach = L.Rows(x, f32(scale)), L.Teacher(tv, ti, x.shape[1], f32(scale))
    want, off = L.loss64(rows, teach)
    R.close(loss, want, off, what="loss")
    R.close(lse, rows.lse, rows.lse_off, what="lse")
    g = torch.ones(1) if dloss is None else dloss
    # (where a row is in parts the fused gradient goes by lse as well)
    d64, off = L.grad64(rows, teach, g)
    _, off2 = L.grad64(rows, teach, g, lse)
    from_lse = L.grad64(rows, teach, g, lse)
    lse_room = (g.double().cpu().abs() * f32(scale)).view(-1, 1) * rows.q * 1.01 * rows.lse_off[:, None].nan_to_num(posinf=0)
    R.close(dx, d64, off + off2 + lse_room, x.dtype, "dx")
    R.close(dx2, from_lse[0], from_lse[1], x.dtype, "dx from lse")


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("m,v", WIDTHS)
def test_distill(m, v, dtype):
    say("distill", m, v, dtype)
    x = logits(m, v, dtype, 11, pad=v % 3)
    for k, scale, t_dtype in ((1, 1.0, F32), (20, 0.5, dtype), (256, 1 / 0.7, BF16)):
        k = min(k, v)
        tv, ti = teacher_of(x, k, 12, t_dtype)
        dloss = torch.rand(m, generator=torch.Generator().manual_seed(13)).cuda() + 0.1
        check_distill(x, tv, ti, scale, {1: None, 20: dloss}.get(k, dloss[:1]))


@pytest.mark.parametrize("v", [60, 3000, 32000, 140000])
def test_distill_lists(v):
    """Lists of other lengths, columns outside the row, columns listed more than once, empty lists."""
    x = logits(8, v, F32, 14)
    tv, ti = teacher_of(x, 30, 15, F32)
    ti = ti.clone()
    ti[0, 5:] = -1
    ti[1] = -1
    ti[2, 3], ti[2, 4], ti[2, 5] = v, 2 ** 31 - 1, -2 ** 31
    ti[3, 10:20] = ti[3, 0:10].clone()
    ti[4] = 7
    tv[5] = NINF
    tv[6, 1:] = NINF
    ti[7, 0], ti[7, 1] = 0, v - 1
    dloss = torch.rand(8, generator=torch.Generator().manual_seed(16)).cuda()
    check_distill(x, tv, ti, 0.7, dloss)
    loss, _, dx, dx2 = run_distill(x, tv, ti, 0.7, dloss)
    assert (loss[[1, 5]] == 0).all() and (dx[[1, 5]] == 0).all() and (dx2[[1, 5]] == 0).all()


@pytest.mark.parametrize("v", [60, 3000, 140000])
def test_distill_masks(v):
    x = logits(6, v, F32, 17)
    tv, ti = teacher_of(x, 10, 18, F32)
    x[0, ti[0, 0].long()] = NINF              # the student rules out what the teacher has: an infinite loss, a finite gradient
    x[1] = NINF                               # nothing left: so here, q = 0
    keep = torch.zeros(v, dtype=torch.bool, device="cuda")
    keep[ti[2].long()] = True
    x[2, ~keep] = NINF
    x[3, ~torch.isin(torch.arange(v, device="cuda"), ti[3].long())] = torch.finfo(F32).min
    dloss = torch.full((6,), 0.5, device="cuda")
    loss, lse, dx, dx2 = run_distill(x, tv, ti, 1.0, dloss)
    assert torch.isinf(loss[:2]).all() and (loss[:2] > 0).all() and torch.isfinite(dx).all() and torch.isfinite(dx2).all()
    check_distill(x, tv, ti, 1.0, dloss)
    for bad in (float("nan"), float("inf")):
        y = x.clone()
        y[4, 3] = bad
        loss, lse, dx, dx2 = run_distill(y, tv, ti, 1.0, dloss)
        assert torch.isnan(loss[4]) and torch.isnan(lse[4]) and torch.isnan(dx[4]).all() and torch.isnan(dx2[4]).all()
        assert torch.isfinite(dx[[2, 3, 5]]).all() and torch.isfinite(loss[[2, 3, 5]]).all()
        t = tv.clone()
        t[5, 2] = bad
        loss, lse, dx, dx2 = run_distill(x, t, ti, 1.0, dloss)
        assert torch.isnan(loss[5]) and torch.isfinite(lse[5]) and torch.isnan(dx[5]).all() and torch.isnan(dx2[5]).all()
        assert torch.isfinite(dx[2:5]).all()


def test_distill_against_differences():
    """Directional differences of the 64-bit loss."""
    m, v, k, scale = 6, 200, 12, f32(0.8)
    x = logits(m, v, F32, 19)
    tv, ti = teacher_of(x, k, 20, F32)
    dloss = torch.rand(m, generator=torch.Generator().manual_seed(21)).cuda()
    _, _, dx, dx2 = run_distill(x, tv, ti, scale, dloss)
    teach = L.Teacher(tv, ti, v, scale)
    x64 = x.double().cpu()

    def total(y):
        return (L.loss64(L.Rows(y, scale), teach)[0] * dloss.double().cpu()).sum()
    for seed in range(4):
        d = torch.randn(m, v, dtype=torch.float64, generator=torch.Generator().manual_seed(seed))
        want = float(total(x64 + 1e-5 * d) - total(x64 - 1e-5 * d)) / 2e-5
        for got in (dx, dx2):
            # second-order remainder 1e-10 / 6 of the third derivative, rounding 1e-16 / 1e-5, the gradient's own 32 bits
            assert abs(float((got.double().cpu() * d).sum()) - want) <= 1e-5 * max(1.0, abs(want))


def test_rows_past_32_bit_offsets():
    m, v, ld = 530, 900, (1 << 20) + 8
    big = torch.empty(m * ld, device="cuda")          # 2.2 GB
    x = big.as_strided((m, v), (ld, 1))
    small = logits(m, v, F32, 22)
    x.copy_(small)
    tok = some_tokens(m, v, 23)
    far, near = run_logprobs(x, tok, 5, 1.0), run_logprobs(small, tok, 5, 1.0)
    assert all(torch.equal(far[k], near[k]) for k in far)
    tv, ti = teacher_of(small, 8, 24, F32)
    loss, lse = torch.empty(m, device="cuda"), torch.empty(m, device="cuda")
    dx = torch.empty_like(small)
    niti.distill_fwd(small, tv, ti, loss, lse=lse, dlogits=dx)
    niti.distill_fwd(x, tv, ti, loss, dlogits=x)
    assert torch.equal(x.contiguous(), dx)
    x.copy_(small)
    niti.distill_bwd(small, tv, ti, lse, None, dx)
    niti.distill_bwd(x, tv, ti, lse, None, x)
    assert torch.equal(x.contiguous(), dx)


@pytest.mark.parametrize("v", [5000, 140000])
def test_stream_and_graph(v):
    m, k = 7, 16
    x, tok = logits(m, v, BF16, 25), some_tokens(m, v, 26)
    tv, ti = (t.contiguous() for t in teacher_of(x, k, 27, F32))
    ws = niti.new_workspace(max(niti.workspace_bytes(niti.OP_TOKEN_LOGPROBS, None, m, v, 9), niti.workspace_bytes(niti.OP_DISTILL_FWD, None, m, v)))
    outs = [torch.empty(m, device="cuda") for _ in range(4)] + [torch.empty(m, 9, device="cuda"), torch.empty(m, 9, dtype=torch.int32, device="cuda"),
                                                                 torch.empty(m, v, dtype=BF16, device="cuda")]

    def step():
        niti.token_logprobs(x, tokens=tok, logp=outs[0], entropy=outs[1], top_logp=outs[4], top_idx=outs[5], ws=ws)
        niti.distill_fwd(x, tv, ti, outs[2], lse=outs[3], dlogits=outs[6], ws=ws)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in range(3):
        x.copy_(logits(m, v, BF16, 30 + seed))
        tok.copy_(some_tokens(m, v, 40 + seed))
        step()
        want = [t.clone() for t in outs]
        for t in outs:
            t.zero_()
        ws.random_(0, 256)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))


def test_refusals():
    x, tok, out = logits(3, 40, F32, 1), some_tokens(3, 40, 2), torch.empty(3, device="cuda")
    top, idx = torch.empty(3, 4, device="cuda"), torch.empty(3, 4, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        niti.token_logprobs(x, tokens=tok)
    with pytest.raises(TypeError):
        niti.token_logprobs(x, tokens=tok.long(), logp=out)
    with pytest.raises(ValueError):
        niti.token_logprobs(x, top_logp=top, top_idx=idx[:, :3])
    with pytest.raises(TypeError):
        niti.token_logprobs(x, top_logp=top, top_idx=[1])
    with pytest.raises(TypeError):
        niti.token_logprobs(x.double(), lse=out)
    for scale in (0.0, -1.0, float("inf"), float("nan")):
        with pytest.raises(niti.NitiError):
            niti.token_logprobs(x, lse=out, scale=scale)
    with pytest.raises(niti.NitiError):
        niti.token_logprobs(x, top_idx=torch.empty(3, 65, dtype=torch.int32, device="cuda"))
    with pytest.raises(niti.NitiError):
        niti.token_logprobs(logits(1, 1 << 21, F32, 1), lse=out[:1])          # no workspace
    with pytest.raises(TypeError):
        niti.distill_fwd(x, top, idx.long(), out)
    with pytest.raises(ValueError):
        niti.distill_fwd(x, top, idx[:, :3], out)
    with pytest.raises(ValueError):
        niti.distill_fwd(x, top, idx, out, dlogits=torch.empty(3, 41, device="cuda"))
    with pytest.raises(niti.NitiError):
        niti.distill_fwd(x, top, idx, out, dloss=out)                         # without dlogits
    with pytest.raises(TypeError):
        niti.distill_bwd(x, top, idx, None, out, x)
    with pytest.raises(TypeError):
        niti.distill_bwd(x, top, idx, out, out, None)
