"""Gated product of int8 rows and its gradients against 64-bit forms (bounds
as in test_gpu_linear.py, carried through the product of the halves)."""
import pytest
import torch

import scaled_ref as R
from helpers import say
from paper_2009_13108_amd import niti
from test_gpu_linear import ACTS, BF16, F16, F32, codes, codes64, floats, row_scales
from test_gpu_linear_kernels import NAMES, launches

pytestmark = pytest.mark.gpu


def near(got, want, bound, dtype, what):
    """scaled_ref.close on the GPU.  A value that rounds past a type's largest, by half a step or more, is stored as an
    infinity: 16-bit floats end at 65504, and a product of two z with a deviation near 73 each may be larger."""
    end = torch.finfo(dtype).max * (1 + R.UNIT[dtype])       # (1 + UNIT) max lies half a step of max's binade above it, or less
    room = bound + R.UNIT[dtype] * (want.abs() + bound) * 1.01 + R.STEP[dtype]
    off = (got.double() - want).abs()
    may = (want.abs() + bound >= end * (1 - R.UNIT[dtype])) & (got == torch.sign(want) * float("inf"))
    must = want.abs() - bound >= end * (1 + R.UNIT[dtype])
    bad = torch.where(must, ~may, ~(off <= room) & ~may)
    assert not bad.any(), "%s: %d of %d off, by up to %g" % (what, int(bad.sum()), off.numel(), float(off[bad].max()))


def forward64(a, b, s_a, s_b, bias, act):
    """(z, its bound, out, its bound) on the operands' device."""
    f = b.shape[0] // 2
    s = (a.double() @ b.double().t()) * (s_a.double().view(-1, 1) * s_b.double().view(1, -1))
    c = bias.double() if bias is not None else torch.zeros(2 * f, dtype=torch.float64, device=s.device)
    z = s + c
    zb = 5 * R.U32 * (s.abs() + c.abs())
    gate, up = z[:, :f], z[:, f:]
    act64 = R.act(act, gate)
    # slopes are at most 1.13; an activation's own evaluation is good to 8 U32 of |z|
    ab = 1.2 * zb[:, :f] + 8 * R.U32 * gate.abs()
    out = act64 * up
    return z, zb, out, ab * (up.abs() + zb[:, f:]) + act64.abs() * zb[:, f:] + 1.01 * R.U32 * out.abs()


def run_forward(m, f, k, dtype, act="silu", bias=True, keep=True, pad=(0, 0), one=(False, False), ws=True, seed=1, kernel=None):
    a, b = codes(m, k, seed, pad[0]), codes(2 * f, k, seed + 1, pad[1])
    s_a, s_b = row_scales(1 if one[0] else m, k, seed + 2) * 4, row_scales(1 if one[1] else 2 * f, 1, seed + 3) * 18
    bi = floats(2 * f, seed=seed + 4, dtype=dtype) if bias else None
    out, io = R.guarded(m, f, dtype)
    z, iz = R.guarded(m, 2 * f, dtype, pad=7)
    space = niti.new_workspace(niti.workspace_bytes(niti.OP_GATED_FWD, None, m, f, k)) if ws else None
    ran = launches(lambda: niti.gated_fwd(a, b, out, s_a, s_b, act=ACTS[act], bias=bi, z=z if keep else None, ws=space))
    if kernel:
        assert ran == [kernel]
    z64, zb, o64, ob = forward64(a, b, s_a, s_b, bi, act)
    near(out, o64, ob, dtype, "out")
    if keep:
        near(z, z64, zb, dtype, "z")
    else:
        assert (z == 77).all()
    io(), iz()


SIZES = [(1, 1, 1), (1, 1, 0), (5, 3, 15), (1, 4096, 4096), (1, 1000, 784), (2, 33, 16), (3, 17, 4099), (8, 128, 64), (16, 16, 64),
         (17, 31, 63), (31, 40, 129), (32, 256, 9216), (33, 64, 1111), (64, 32, 64), (65, 65, 65), (100, 84, 120), (127, 127, 48),
         (128, 64, 128), (129, 257, 4096), (200, 10, 8192), (256, 128, 80), (257, 150, 272), (500, 500, 304), (1000, 750, 1111),
         (1031, 384, 512), (2048, 512, 640), (1, 1, 131071), (1500, 1600, 1803)]


@pytest.mark.parametrize("m,f,k", SIZES)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_forward(m, f, k, dtype):
    say("gated_fwd", m, f, k, dtype)
    run_forward(m, f, k, dtype, act="gelu" if dtype is F32 else "silu")
    run_forward(m, f, k, dtype, act="relu", bias=False, keep=False, ws=False)


@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("m,f,k", [(1, 200, 256), (40, 72, 96), (300, 260, 128)])
def test_forward_epilogues(m, f, k, dtype, act):
    say("gated_fwd", m, f, k, dtype, act)
    for bias in (False, True):
        for keep in (False, True):
            run_forward(m, f, k, dtype, act, bias, keep)
    for one in ((True, False), (False, True), (True, True)):
        run_forward(m, f, k, dtype, act, one=one)


@pytest.mark.parametrize("pad", [(0, 3), (1, 0), (5, 7), (16, 48), (16, 1)])
@pytest.mark.parametrize("m,f,k", [(1, 130, 144), (7, 96, 100), (70, 130, 256), (300, 256, 512), (520, 520, 1000)])
def test_forward_strides(m, f, k, pad):
    say("gated_fwd strides", m, f, k, pad)
    run_forward(m, f, k, BF16, pad=pad)


RING64, RING128, DEEP128, RING256 = "64,128,3,2,2,128", "128,128,2,4,2,128", "128,128,4,4,2,128", "256,256,4,2,4,64"

# rows, columns, sum, padding of the operands' rows, kernel without z, kernel with it (None: the same)
CASES = [
    (4001, 2001, 272, (0, 0), "ring:" + RING256, None), (3841, 2045, 2064, (0, 16), "ring:" + RING256, None),
    (4001, 1999, 1003, (1, 2), "ring:" + RING256, None),                                                     # rows copied first
    (4001, 2001, 16, (0, 0), "ring:" + RING128, None), (4001, 2001, 80, (16, 0), "ring:" + RING128, None),
    (2100, 1051, 1040, (0, 0), "ring:" + RING128, None), (2100, 1051, 515, (3, 0), "ring:" + RING128, None),
    (257, 10001, 160, (0, 48), "ring:" + RING128, None),
    (2000, 751, 528, (0, 0), "ring:" + DEEP128, None), (1024, 1100, 2048, (16, 16), "ring:" + DEEP128, None),
    (1500, 751, 304, (0, 0), "ring:" + DEEP128, "ring:" + RING64), (1000, 751, 16, (0, 0), "ring:" + DEEP128, "ring:" + RING64),
    (999, 753, 400, (48, 0), "ring:" + RING64, None), (700, 700, 1024, (0, 0), "ring:" + RING64, None),
    (1000, 751, 97, (2, 5), "any", None), (1000, 751, 100, (4, 8), "any", None), (1500, 751, 300, (1, 1), "any", None),
    (1, 1001, 260, (4, 0), "small:2,2,0", "small:1,2,0"), (300, 500, 4100, (0, 0), "small:2,2,0", None),
    (257, 257, 148, (0, 4), "small:2,2,0", "small:1,2,0"),
    (1, 1001, 259, (1, 0), "small:1,2,1", None), (257, 257, 143, (0, 2), "small:1,2,1", None), (300, 500, 4096, (1, 0), "small:2,2,1", None),
]


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("m,f,k,pad,without,with_z", CASES)
def test_kernel(m, f, k, pad, without, with_z, dtype):
    """Each kernel at ragged sizes that the choice gives it: the timing records say which ran."""
    say("gated kernel", m, f, k, pad, without, with_z, dtype)

    def label(kernel):
        kind, _, args = kernel.partition(":")
        return "linear_%s_kernel<%s,%spairs>" % (kind, NAMES[dtype], args + "," if args else "")
    run_forward(m, f, k, dtype, act="silu", keep=False, pad=pad, kernel=label(without))
    run_forward(m, f, k, dtype, act="gelu", keep=True, pad=pad, kernel=label(with_z or without))


def test_forward_special_values():
    m, f, k = 70, 90, 96
    a, b = codes(m, k, 1), codes(2 * f, k, 2)
    s_a, s_b = row_scales(m, k, 3), row_scales(2 * f, 1, 4)
    s_a[5] = float("nan")                                   # a row that was not finite
    a[6] = 0                                                # an empty row: act(bias) * bias
    bias = floats(2 * f, seed=5)
    bias[3] = float("-inf")
    out, z = torch.empty(m, f, device="cuda"), torch.empty(m, 2 * f, device="cuda")
    for act in ("relu", "gelu", "silu"):
        niti.gated_fwd(a, b, out, s_a, s_b, act=ACTS[act], bias=bias, z=z)
        o = out.cpu()
        assert torch.isnan(o[5]).all()
        row = torch.tensor([i for i in range(m) if i != 5])
        assert torch.isfinite(o[row]).all() and (o[row, 3].abs() < 1e-30).all()     # act(-inf) is 0
        assert torch.equal(z[6].cpu(), bias.cpu())
    niti.gated_fwd(a[:0], b, out[:0], s_a[:0], s_b)
    niti.gated_fwd(a, b[:0], out[:, :0], s_a, s_b[:0])
    one = s_a[:1]
    niti.gated_fwd(a[:, :0], b[:, :0], out, one, one, bias=bias * 0 + 2, act=niti.ACT_RELU)
    assert torch.isnan(out[:, 3]).all()                     # (its bias: minus infinity times 0)
    out[:, 3] = 4
    assert (out == 4).all()


def test_forward_past_32_bit_offsets():
    """Rows far apart: operands and results beyond 2^31 bytes, b's partners beyond them from its gates."""
    m, f, k = 600, 300, 64
    ld = (1 << 22) - 16
    small_a, small_b = codes(m, k, 1), codes(2 * f, k, 2)
    s_a, s_b = row_scales(m, k, 3), row_scales(2 * f, 1, 4)
    want, out, z = (torch.empty(m, n, device="cuda") for n in (f, f, 2 * f))
    niti.gated_fwd(small_a, small_b, want, s_a, s_b, z=z)
    big = torch.empty(2 * f * ld, dtype=torch.int8, device="cuda")          # 2.5 GB
    b = big.as_strided((2 * f, k), (ld, 1))
    b.copy_(small_b)
    niti.gated_fwd(small_a, b, out, s_a, s_b)
    assert torch.equal(out, want)
    wide = big.view(F32)[: m * (ld // 4)].as_strided((m, 2 * f), (ld // 4, 1))
    niti.gated_fwd(small_a, small_b, out, s_a, s_b, z=wide)
    assert torch.equal(wide.contiguous(), z)


def halves64(dy, z, act):
    """dz, and the magnitudes that a slope's or an activation's own error goes with."""
    f = dy.shape[1]
    gate, up = z[:, :f], z[:, f:]
    dz = torch.cat([dy * up * R.slope(act, gate), dy * R.act(act, gate)], dim=1)
    return dz, torch.cat([(dy * up).abs(), (dy * gate).abs()], dim=1)


def backward64(dy, z, act, a, b, s_a, s_b, u=None, v=None):
    dy, z, a, b = (t.double().cpu() for t in (dy, z, a, b))
    s_a, s_b = s_a.double().cpu().expand(a.shape[0]), s_b.double().cpu().expand(b.shape[0])
    dz, mag = halves64(dy, z, act)
    x = dz * s_b
    r = R.scales(x)
    p, near_p = codes64(x, r, u)
    da = r[:, None] * (p @ b)
    # as test_gpu_linear.backward64, two roundings more in dz
    dab = 44 * R.U32 * da.abs() + r[:, None] * (near_p.double() @ b.abs()) + 8 * R.U32 * R.scales(mag * s_b)[:, None] * (p @ b).abs()
    x = (dz * s_a[:, None]).t()
    c = R.scales(x)
    q, near_q = codes64(x, c, v)
    db = c[:, None] * (q @ a)
    dbb = 44 * R.U32 * db.abs() + c[:, None] * (near_q.double() @ a.abs()) + \
        8 * R.U32 * R.scales((mag * s_a[:, None]).t())[:, None] * (q @ a).abs()
    return da, dab, db, dbb, dz.sum(dim=0), 84 * R.U32 * dz.abs().sum(dim=0) + 8 * R.U32 * mag.sum(dim=0)


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("m,f,k,act,mode", [
    (1, 1, 1, "none", "rtn"), (1, 300, 200, "silu", "sr"), (5, 33, 17, "gelu", "rtn"), (64, 64, 64, "relu", "sr"),
    (100, 127, 130, "silu", "rtn"), (129, 500, 784, "gelu", "sr"), (700, 128, 256, "none", "sr"), (1100, 300, 96, "silu", "rtn"),
    (31, 1025, 64, "relu", "rtn"), (40, 2049, 48, "none", "rtn"), (20, 9000, 40, "silu", "sr"), (513, 256, 512, "gelu", "rtn"),
    (270, 265, 96, "silu", "rtn"), (500, 8, 64, "relu", "sr"), (33, 7, 20, "silu", "sr")])
def test_backward(m, f, k, act, mode, dtype):
    say("gated_bwd", m, f, k, act, mode, dtype)
    a, b = codes(m, k, 1, pad=k % 3), codes(2 * f, k, 2)
    s_a, s_b = row_scales(m, k, 3), row_scales(2 * f, 1, 4)
    dy, z = floats(m, f, seed=5, dtype=dtype), floats(m, 2 * f, seed=6, dtype=dtype, scale=1.5)
    da, ia = R.guarded(m, k, dtype)
    db, ib = R.guarded(2 * f, k, dtype)
    dbias = torch.empty(2 * f, device="cuda")
    ws = niti.new_workspace(niti.workspace_bytes(niti.OP_GATED_BWD, None, m, f, k))
    ws.random_(0, 256)
    kw = dict(act=ACTS[act], mode=niti.SR if mode == "sr" else niti.RTN, seed=77, call=5)
    niti.gated_bwd(dy, z, a, b, s_a, s_b, ws, da=da, db=db, dbias=dbias, **kw)
    u = v = None
    if mode == "sr":
        r = R.draws(77, 5, m * 2 * f)
        u, v = R.field(r, 40, 24).view(m, 2 * f), R.field(r, 8, 24).view(m, 2 * f).t()
    wa, ba, wb, bb, wd, bd = backward64(dy, z, act, a, b, s_a, s_b, u, v)
    R.close(da, wa, ba, dtype, "da")
    R.close(db, wb, bb, dtype, "db")
    R.close(dbias, wd, bd, what="dbias")
    ia(), ib()
    # each alone gives the same, and so do strided operands
    ws.random_(0, 256)
    one, two, three = torch.empty(m, k, dtype=dtype, device="cuda"), torch.empty(2 * f, k, dtype=dtype, device="cuda"), torch.empty_like(dbias)
    wide_z, wide_dy = (torch.nn.functional.pad(t, (0, 5))[:, :t.shape[1]] for t in (z, dy))
    niti.gated_bwd(wide_dy, wide_z, a, b, s_a, s_b, ws, da=one, **kw)
    niti.gated_bwd(dy, wide_z, a, b, s_a, s_b, ws, db=two, **kw)
    niti.gated_bwd(wide_dy, z, a, b, s_a, s_b, ws, dbias=three, **kw)
    assert torch.equal(one, da) and torch.equal(two, db) and torch.equal(three, dbias)


def test_backward_against_differences():
    """Directional differences of the 64-bit forward pass; the int8 products are
    off by at most half a step of the error's codes."""
    m, f, k = 24, 20, 56
    a, b = codes(m, k, 1), codes(2 * f, k, 2)
    s_a, s_b = row_scales(m, k, 3), row_scales(2 * f, 1, 4)
    dy, bias = floats(m, f, seed=5), floats(2 * f, seed=6)
    z, out = torch.empty(m, 2 * f, device="cuda"), torch.empty(m, f, device="cuda")
    da, db, dbias = torch.empty(m, k, device="cuda"), torch.empty(2 * f, k, device="cuda"), torch.empty(2 * f, device="cuda")
    ws = niti.new_workspace(niti.workspace_bytes(niti.OP_GATED_BWD, None, m, f, k))
    for act in ACTS:
        niti.gated_fwd(a, b, out, s_a, s_b, bias=bias, act=ACTS[act], z=z)
        niti.gated_bwd(dy, z, a, b, s_a, s_b, ws, act=ACTS[act], da=da, db=db, dbias=dbias)
        av, bv = a.double().cpu() * s_a.double().cpu()[:, None], b.double().cpu() * s_b.double().cpu()[:, None]
        bias64, dy64 = bias.double().cpu(), dy.double().cpu()

        def loss(x, w, c):
            y = x @ w.t() + c
            return (R.act(act, y[:, :f]) * y[:, f:] * dy64).sum()
        dz, _ = halves64(dy64, z.double().cpu(), act)
        half_a = 0.5 * R.scales(dz * s_b.double().cpu())[:, None] * b.double().cpu().abs().sum(dim=0)
        half_b = 0.5 * R.scales((dz * s_a.double().cpu()[:, None]).t())[:, None] * a.double().cpu().abs().sum(dim=0)
        for seed in range(3):
            g = torch.Generator().manual_seed(seed)
            va, vb = (torch.randn(t.shape, generator=g, dtype=torch.float64) for t in (av, bv))
            vc = torch.randn(2 * f, generator=g, dtype=torch.float64)
            e = 1e-6
            for got, v, room, want in (
                    (da, va, half_a, (loss(av + e * va, bv, bias64) - loss(av - e * va, bv, bias64)) / (2 * e)),
                    (db, vb, half_b, (loss(av, bv + e * vb, bias64) - loss(av, bv - e * vb, bias64)) / (2 * e)),
                    (dbias, vc, torch.zeros(2 * f, dtype=torch.float64),
                     (loss(av, bv, bias64 + e * vc) - loss(av, bv, bias64 - e * vc)) / (2 * e))):
                off = abs(float((got.double().cpu() * v).sum() - want))
                assert off <= float((room * v.abs()).sum()) * 1.01 + 1e-4 * max(1.0, abs(float(want))), (act, off)


def test_backward_special_rows():
    m, f, k = 50, 35, 32
    a, b = codes(m, k, 1), codes(2 * f, k, 2)
    s_a, s_b = row_scales(m, k, 3), row_scales(2 * f, 1, 4)
    dy, z = floats(m, f, seed=5), floats(m, 2 * f, seed=6)
    dy[3], dy[:, 4] = 0, 0
    da, db, dbias = torch.empty(m, k, device="cuda"), torch.empty(2 * f, k, device="cuda"), torch.empty(2 * f, device="cuda")
    ws = niti.new_workspace(niti.workspace_bytes(niti.OP_GATED_BWD, None, m, f, k))
    niti.gated_bwd(dy, z, a, b, s_a, s_b, ws, da=da, db=db, dbias=dbias)
    assert (da[3] == 0).all() and (db[4] == 0).all() and (db[f + 4] == 0).all() and float(dbias[4]) == 0 == float(dbias[f + 4])
    assert torch.isfinite(da).all() and torch.isfinite(db).all()
    dy[7, 9] = float("inf")
    niti.gated_bwd(dy, z, a, b, s_a, s_b, ws, da=da, db=db, dbias=dbias)
    assert torch.isnan(da[7]).all() and torch.isnan(db[[9, f + 9]]).all() and not torch.isfinite(dbias[[9, f + 9]]).any()
    ok_m, ok_n = [i for i in range(m) if i != 7], [i for i in range(2 * f) if i not in (9, f + 9)]
    assert torch.isfinite(da[ok_m]).all() and torch.isfinite(db[ok_n]).all() and torch.isfinite(dbias[ok_n]).all()
    db.fill_(5), dbias.fill_(5)
    niti.gated_bwd(dy[:0], z[:0], a[:0], b, s_a[:0], s_b, ws, da=da[:0], db=db, dbias=dbias)
    assert (db == 0).all() and (dbias == 0).all()


def test_other_device_stream_and_graph():
    """On a stream of the caller's, captured and replayed with other inputs in the same memory."""
    m, f, k = 130, 200, 257
    a, b = codes(m, k, 1), codes(2 * f, k, 2)
    s_a, s_b = row_scales(m, k, 3), row_scales(2 * f, 1, 4)
    dy = floats(m, f, seed=5, dtype=BF16)
    z, out = torch.empty(m, 2 * f, dtype=BF16, device="cuda"), torch.empty(m, f, dtype=BF16, device="cuda")
    da, db, dbias = (torch.empty(r, c, dtype=BF16, device="cuda") for r, c in ((m, k), (2 * f, k), (1, 1)))
    dbias = torch.empty(2 * f, device="cuda")
    ws = niti.new_workspace(max(niti.workspace_bytes(op, None, m, f, k) for op in (niti.OP_GATED_FWD, niti.OP_GATED_BWD)))

    def step():
        niti.gated_fwd(a, b, out, s_a, s_b, z=z, ws=ws)
        niti.gated_bwd(dy, z, a, b, s_a, s_b, ws, da=da, db=db, dbias=dbias)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in range(3):
        a.copy_(codes(m, k, 10 + seed))
        dy.copy_(floats(m, f, seed=20 + seed, dtype=BF16))
        step()
        want = [t.clone() for t in (out, z, da, db, dbias)]
        for t in (out, z, da, db, dbias):
            t.zero_()
        ws.random_(0, 256)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip((out, z, da, db, dbias), want))


def test_refusals():
    a, b, out = codes(4, 16, 1), codes(12, 16, 2), torch.empty(4, 6, device="cuda")
    s_a, s_b = torch.ones(4, device="cuda"), torch.ones(12, device="cuda")
    with pytest.raises(ValueError):
        niti.gated_fwd(a, codes(11, 16, 2), out, s_a, s_b)
    with pytest.raises(ValueError):
        niti.gated_fwd(a, b, out, s_a, s_b[:6])
    with pytest.raises(ValueError):
        niti.gated_fwd(a, b, out, s_a, s_b, z=torch.empty(4, 6, device="cuda"))
    with pytest.raises(TypeError):
        niti.gated_fwd(a.float(), b, out, s_a, s_b)
    with pytest.raises(TypeError):
        niti.gated_fwd(a, None, out, s_a, s_b)
    with pytest.raises(niti.NitiError):
        niti.gated_fwd(a, b, out, s_a, s_b, act=9)
    z, da = torch.empty(4, 12, device="cuda"), torch.empty(4, 16, device="cuda")
    with pytest.raises(niti.NitiError):
        niti.gated_bwd(out, z, a, b, s_a, s_b, niti.new_workspace(256), da=da)      # workspace too small
    ws = niti.new_workspace(niti.workspace_bytes(niti.OP_GATED_BWD, None, 4, 6, 16))
    with pytest.raises(TypeError):
        niti.gated_bwd(out, None, a, b, s_a, s_b, ws, da=da)
    with pytest.raises(niti.NitiError):
        niti.gated_bwd(out, z, a, b, s_a, s_b, ws, da=da, mode=niti.PSR)
