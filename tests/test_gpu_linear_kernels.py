"""Each kernel that a product of int8 rows may run, at ragged sizes that the choice
gives it: the timing records say which ran, and a change of the choice that
takes a kernel's cases away shows here.  64-bit forms as in test_gpu_linear.py, on the GPU."""
import pytest
import torch

import scaled_ref as R
from helpers import say
from paper_2009_13108_amd import niti
from test_gpu_linear import ACTS, BF16, F16, F32, backward64, codes, floats, row_scales

pytestmark = pytest.mark.gpu
NAMES = {F32: "f32", BF16: "bf16", F16: "f16"}


def launches(call):
    """Labels of the product kernels and joins of a call."""
    niti.timing_enable(True)
    call()
    niti.timing_enable(False)
    torch.cuda.synchronize()
    return [name for fam, name, _ in niti.timing_records() if fam in (niti.TIMING_KERNEL, niti.TIMING_SUM)]


def forward64(a, b, s_a, s_b, bias, act, res):
    """(z, its bound, out, its bound), as test_gpu_linear.forward64 derives them."""
    s = (a.double() @ b.double().t()) * (s_a.double().view(-1, 1) * s_b.double().view(1, -1))
    z = s + bias.double()
    zb = 5 * R.U32 * (s.abs() + bias.double().abs())
    out = {"relu": lambda: z.clamp(min=0), "silu": lambda: z * torch.sigmoid(z)}[act]()
    if res is not None:
        out = out + res.double()
    return z, zb, out, 1.2 * zb + 8 * R.U32 * z.abs() + R.U32 * out.abs()


def near(got, want, bound, dtype, what):
    """scaled_ref.close on the GPU, for finite values."""
    room = bound + R.UNIT[dtype] * (want.abs() + bound) * 1.01 + R.STEP[dtype]
    off = (got.double() - want).abs()
    assert torch.isfinite(got).all() and (off <= room).all(), "%s: %d of %d off, by up to %g" % (
        what, int((off > room).sum()), off.numel(), float(off.max()))


RING64, RING128, DEEP128, RING256 = "64,64,3,2,2,128", "128,128,2,4,2,128", "128,128,4,4,2,128", "256,256,4,2,4,64"

# rows, columns, sum, padding of the operands' rows, kernel
CASES = [
    (4001, 3999, 16, (0, 0), "ring:" + RING256), (4001, 3999, 80, (16, 0), "ring:" + RING256),     # one and two steps of four stages
    (3999, 4001, 144, (0, 48), "ring:" + RING256), (4001, 3999, 272, (0, 0), "ring:" + RING256),
    (3841, 4090, 2064, (0, 0), "ring:" + RING256), (4001, 3999, 1003, (1, 2), "ring:" + RING256),  # rows copied first
    (2101, 2097, 16, (0, 16), "ring:" + RING128), (2100, 2101, 1040, (0, 0), "ring:" + RING128), (257, 20001, 160, (0, 0), "ring:" + RING128),
    (2100, 2101, 515, (3, 0), "ring:" + RING128),
    (2000, 1501, 528, (0, 0), "ring:" + DEEP128), (1500, 1501, 784, (16, 16), "ring:" + DEEP128),
    (1000, 1501, 16, (0, 0), "ring:" + RING64), (1500, 1501, 304, (0, 0), "ring:" + RING64), (999, 1503, 400, (48, 0), "ring:" + RING64),
    (1000, 1501, 97, (2, 5), "any"), (1000, 1501, 100, (4, 8), "any"), (1500, 1501, 300, (1, 1), "any"),
    (1, 1001, 260, (4, 0), "small:1,1,0"), (257, 513, 148, (0, 4), "small:1,2,0"), (300, 1000, 4100, (0, 0), "small:2,2,0"),
    (1, 1001, 259, (1, 0), "small:1,1,1"), (257, 513, 143, (0, 2), "small:1,2,1"), (300, 1000, 4096, (1, 0), "small:2,2,1"),
]


def label(kernel, dtype):
    kind, _, args = kernel.partition(":")
    return "linear_%s_kernel<%s%s>" % (kind, NAMES[dtype], "," + args if args else "")


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("m,n,k,pad,kernel", CASES)
def test_kernel(m, n, k, pad, kernel, dtype):
    say("linear kernel", m, n, k, pad, kernel, dtype)
    a, b = codes(m, k, 1, pad[0]), codes(n, k, 2, pad[1])
    s_a, s_b = row_scales(m, k, 3) * 4, row_scales(n, 1, 4) * 18
    bias, res = floats(n, seed=5, dtype=dtype), floats(m, n, seed=6, dtype=dtype)
    ws = niti.new_workspace(niti.workspace_bytes(niti.OP_LINEAR_FWD, None, m, n, k))
    out, io = R.guarded(m, n, dtype)
    z, iz = R.guarded(m, n, dtype, pad=7)
    for keep, add, act in ((True, True, "silu"), (False, False, "relu"), (True, False, "relu"), (False, True, "silu")):
        out.fill_(7), z.fill_(7)
        kw = dict(bias=bias, act=ACTS[act], res=res if add else None, z=z if keep else None, ws=ws)
        assert launches(lambda: niti.linear_fwd(a, b, out, s_a, s_b, **kw)) == [label(kernel, dtype)]
        wz, zb, wo, ob = forward64(a, b, s_a, s_b, bias, act, res if add else None)
        near(out, wo, ob, dtype, "out")
        if keep:
            near(z, wz, zb, dtype, "z")
        else:
            assert (z == 7).all()
    io(), iz()


@pytest.mark.parametrize("m,n,k,parts", [(140, 130, 131056, "ring:" + RING64), (60, 30, 20000, "ring:" + RING64),
                                         (140, 130, 131071, "any"), (20, 40, 131057, "any")])
def test_sums_of_parts(m, n, k, parts):
    """Parts of long sums side by side, at the ends of what int32 holds: exactly."""
    say("linear parts", m, n, k)
    a = torch.full((m, k), -128, dtype=torch.int8, device="cuda")
    b = torch.full((n, k), -128, dtype=torch.int8, device="cuda")
    b[1:2] = 127
    b[2, : k // 2] = 127            # parts of opposite signs
    one, out = torch.ones(1, device="cuda"), torch.empty(m, n, device="cuda")
    ws = niti.new_workspace(niti.workspace_bytes(niti.OP_LINEAR_FWD, None, m, n, k))
    ran = launches(lambda: niti.linear_fwd(a, b, out, one, one, ws=ws))
    assert ran == [label(parts, F32).replace("f32", "i32"), "linear_join_kernel<f32>"]
    want = torch.full((m, n), float(k * 16384))
    want[:, 1] = -float(k * 128 * 127)
    want[:, 2] = float((k - k // 2) * 16384 - k // 2 * 128 * 127)
    assert torch.equal(out.cpu(), want.float())


@pytest.mark.parametrize("m,n,k,kernel", [(4001, 3999, 144, "ring:" + RING256), (1000, 1501, 144, "ring:" + RING64),
                                          (2101, 2097, 144, "ring:" + RING128), (1000, 1501, 100, "any")])
def test_rows_far_apart(m, n, k, kernel):
    """Operands, residual, z and result side by side in rows of nearly 4 MiB: offsets past 32 bits in all of them."""
    say("linear far rows", m, n, k, kernel)
    ld = (1 << 22) - 16
    big = torch.empty(max(m, n) * ld, dtype=torch.int8, device="cuda")
    half = big.view(BF16)

    def rows(r, c, at, whole):   # at: bytes into each row
        return whole.as_strided((r, c), (ld // whole.element_size(), 1), at // whole.element_size())
    a, b = rows(m, k, 0, big), rows(n, k, 1024, big)
    res, z, out = (rows(m, n, at, half) for at in (1 << 14, 1 << 16, 1 << 18))
    sa, sb = codes(m, k, 1), codes(n, k, 2)
    a.copy_(sa), b.copy_(sb)
    s_a, s_b = row_scales(m, k, 3) * 4, row_scales(n, 1, 4) * 18
    bias, r = floats(n, seed=5, dtype=BF16), floats(m, n, seed=6, dtype=BF16)
    res.copy_(r)
    kw = dict(bias=bias, act=ACTS["silu"])
    z2, o2 = torch.empty(m, n, dtype=BF16, device="cuda"), torch.empty(m, n, dtype=BF16, device="cuda")
    assert launches(lambda: niti.linear_fwd(a, b, out, s_a, s_b, res=res, z=z, **kw)) == [label(kernel, BF16)]
    niti.linear_fwd(sa, sb, o2, s_a, s_b, res=r, z=z2, **kw)
    assert torch.equal(out, o2) and torch.equal(z, z2)
    assert torch.equal(res, r) and torch.equal(a, sa) and torch.equal(b, sb)


PAIRS = [
    # both small in one launch; both of 64 x 64 tiles in one; apart, by large tiles
    (40, 100, 96, ["linear_small_pair_kernel<bf16,1,1>"]),
    (500, 700, 250, ["linear_small_pair_kernel<bf16,2,2>"]),
    (1030, 1100, 700, ["linear_ring_pair_kernel<bf16,64,64,3,2,2,128>"]),
    (4001, 160, 3999, ["linear_ring_kernel<bf16,64,64,3,2,2,128>", "linear_ring_kernel<bf16,256,256,4,2,4,64>"]),
    (2100, 2101, 2090, ["linear_ring_kernel<bf16,128,128,2,4,2,128>"] * 2),
]


@pytest.mark.parametrize("mode", [niti.RTN, niti.SR])
@pytest.mark.parametrize("m,n,k,kernels", PAIRS)
def test_gradient_products(m, n, k, kernels, mode):
    say("linear gradients", m, n, k, mode)
    a, b = codes(m, k, 1, pad=3), codes(n, k, 2)
    s_a, s_b = row_scales(m, k, 3), row_scales(n, 1, 4)
    dy, zz = floats(m, n, seed=5, dtype=BF16), floats(m, n, seed=6, dtype=BF16, scale=1.5)
    (da, ia), (db, ib) = R.guarded(m, k, BF16), R.guarded(n, k, BF16)
    dbias = torch.empty(n, device="cuda")
    ws = niti.new_workspace(niti.workspace_bytes(niti.OP_LINEAR_BWD, None, m, n, k))
    ran = launches(lambda: niti.linear_bwd(dy, a, b, s_a, s_b, ws, z=zz, act=ACTS["silu"], da=da, db=db, dbias=dbias, mode=mode,
                                           seed=21, call=4))
    assert ran == kernels
    u = v = None
    if mode == niti.SR:
        r = R.draws(21, 4, m * n)
        u, v = R.field(r, 40, 24).view(m, n), R.field(r, 8, 24).view(m, n).t()
    wa, ba, wb, bb, wd, bd = backward64(dy, zz, "silu", a, b, s_a, s_b, u, v)
    R.close(da, wa, ba, BF16, "da")
    R.close(db, wb, bb, BF16, "db")
    R.close(dbias, wd, bd, what="dbias")
    ia(), ib()
