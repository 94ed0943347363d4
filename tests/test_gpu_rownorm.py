"""Root-mean-square norm with int8 rows, its gradients, and the quantisation
of rows, against 64-bit forms (tests/scaled_ref.py has the bounds)."""
import pytest
import torch

import scaled_ref as R
from helpers import say
from paper_2009_13108_amd import niti

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def data(m, d, dtype, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(m, d, generator=g) * scale).to(dtype).cuda()


SHAPES = [(1, 1), (1, 4096), (3, 7), (5, 8), (2, 64), (4, 511), (9, 513), (130, 1111), (6, 2048), (7, 2049), (3, 4100), (33, 784),
          (2, 8192), (3, 8193), (2, 16385), (2, 32768), (2, 40001)]


def forward64(x, res, gain, eps):
    h = x.double().cpu() + (res.double().cpu() if res is not None else 0)
    rstd = 1 / torch.sqrt((h * h).mean(dim=1) + eps)
    return h, rstd, h * rstd[:, None] * gain.double().cpu()


# y: rstd off by less than (42 / 2 + 4) U32, two products more
Y_REL = 32 * R.U32


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("m,d", SHAPES)
def test_forward(m, d, dtype):
    say("rmsnorm_fwd", m, d, dtype)
    x, res = data(m, d, dtype, 1), data(m, d, dtype, 2)
    gain = (1 + 0.1 * data(1, d, F32, 3)[0]).to(BF16 if dtype is F16 else F32)   # a type of its own
    eps = 1e-5
    h, rstd, y = forward64(x, res, gain, eps)
    oh, ih = R.guarded(m, d, dtype)
    oy, iy = R.guarded(m, d, dtype, pad=3)
    oq, iq = R.guarded(m, d, torch.int8, pad=5)
    scale, orstd = torch.zeros(m, device="cuda"), torch.zeros(m, device="cuda")
    niti.rmsnorm_fwd(x, gain, res=res, h=oh, y=oy, q=oq, scale=scale, rstd=orstd, eps=eps)
    R.close(oh, h, R.U32 * h.abs(), dtype, "h")
    R.close(orstd, rstd, 25 * R.U32 * rstd, what="rstd")
    s = R.scales(y)
    R.close(scale, s, (Y_REL + 2 * R.U32) * s, what="scale")
    R.check_codes(oq, y, s)
    # y: the codes' values, one product and one rounding
    R.close(oy, oq.double().cpu() * scale.double().cpu()[:, None], R.U32 * (127 * scale.double().cpu()[:, None]), dtype, "y of codes")
    ih(), iy(), iq()
    # without codes: y itself; without a residual
    _, _, y = forward64(x, None, gain, eps)
    niti.rmsnorm_fwd(x, gain, y=oy, eps=eps)
    R.close(oy, y, Y_REL * y.abs(), dtype, "y")
    iy()


def test_forward_special_rows():
    d = 300
    x = data(8, d, F32, 5)
    x[0] = 0                                   # empty (a padding token): zeros, a finite scale
    x[1, 7] = float("nan")
    x[2, 9] = float("inf")
    x[3] *= 1e30                               # its squares leave the 32-bit range
    x[4] *= 1e-30                              # its squares vanish; eps decides
    x[5, 1:] = 0
    x[6] = torch.finfo(F32).max
    x[7] = -torch.finfo(F32).max
    gain = torch.ones(d, device="cuda")
    q, scale = torch.full((8, d), 5, dtype=torch.int8, device="cuda"), torch.zeros(8, device="cuda")
    y, rstd = torch.empty_like(x), torch.zeros(8, device="cuda")
    niti.rmsnorm_fwd(x, gain, y=y, q=q, scale=scale, rstd=rstd, eps=1e-6)
    q, scale, y = q.cpu(), scale.cpu(), y.cpu()
    assert (q[0] == 0).all() and (y[0] == 0).all() and abs(float(scale[0]) / (R.TINY / 127) - 1) < 1e-6
    assert (q[1:3] == 0).all() and torch.isnan(scale[1:3]).all() and torch.isnan(y[1:3]).all()
    assert (q[6] == 127).all() and (q[7] == -127).all()
    _, r64, y64 = forward64(x, None, gain, 1e-6)
    for i in (3, 4, 5, 6, 7):
        s = R.scales(y64[i:i + 1])
        R.check_codes(q[i:i + 1], y64[i:i + 1], s, what="row %d" % i)
        R.close(scale[i:i + 1], s, 40 * R.U32 * s, what="scale of row %d" % i)
    # reciprocal norms below the normal range lose bits as any 32-bit value there
    R.close(rstd[3:8], r64[3:8], 40 * R.U32 * r64[3:8] + 2.0 ** -149, what="rstd")


def test_forward_in_place_and_broadcast():
    x, row = data(37, 1000, BF16, 7), data(1, 1000, BF16, 8)
    gain = torch.ones(1000, device="cuda")
    h, y = torch.empty_like(x), torch.empty_like(x)
    niti.rmsnorm_fwd(x, gain, res=row.repeat(37, 1), h=h, y=y)
    x2, y2 = x.clone(), torch.empty_like(x)
    niti.rmsnorm_fwd(x2, gain, res=row.expand(37, 1000), h=x2, y=y2)      # stride 0; h over x
    assert torch.equal(x2, h) and torch.equal(y2, y)
    x3 = x.clone()
    niti.rmsnorm_fwd(x3, gain, res=row.expand(37, 1000), y=x3)            # y over x
    assert torch.equal(x3, y)
    big = data(3, 40000, BF16, 9)                                        # the kernel for long rows
    gain = torch.ones(40000, device="cuda")
    y, b2 = torch.empty_like(big), big.clone()
    niti.rmsnorm_fwd(big, gain, y=y)
    niti.rmsnorm_fwd(b2, gain, y=b2)
    assert torch.equal(b2, y)


def test_no_rows():
    gain = torch.ones(16, device="cuda")
    x = torch.empty(0, 16, device="cuda")
    niti.rmsnorm_fwd(x, gain, y=torch.empty_like(x))
    niti.quantize_rows(x, torch.empty(0, 16, dtype=torch.int8, device="cuda"), torch.empty(0, device="cuda"))
    dgain = torch.full((16,), 3.0, device="cuda")
    niti.rmsnorm_bwd(x, x, gain, torch.empty(0, device="cuda"), torch.empty_like(x), dgain)
    assert (dgain == 0).all()


def backward64(dy, h, gain, rstd, dh):
    dy, h, gain, rstd = (t.double().cpu() for t in (dy, h, gain, rstd))
    xh = h * rstd[:, None]
    t = dy * gain
    dx = rstd[:, None] * (t - xh * (t * xh).mean(dim=1, keepdim=True))
    # (42 + 8) U32 on each term of the difference
    bound = 50 * R.U32 * rstd[:, None] * (t.abs() + xh.abs() * (t * xh).abs().mean(dim=1, keepdim=True))
    if dh is not None:
        dx = dx + dh.double().cpu()
        bound = bound + R.U32 * dx.abs()
    rows = dy * xh
    return dx, bound, rows.sum(dim=0), rows.abs().sum(dim=0)


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("m,d", SHAPES + [(2100, 96), (1030, 2500)])
def test_backward(m, d, dtype):
    say("rmsnorm_bwd", m, d, dtype)
    h, dy, dh = data(m, d, dtype, 11), data(m, d, dtype, 12, 0.1), data(m, d, dtype, 13, 0.1)
    gain = 1 + 0.1 * data(1, d, F32, 14)[0]
    rstd = (1 / torch.sqrt(h.double().square().mean(dim=1) + 1e-6)).float()
    ws = niti.new_workspace(niti.workspace_bytes(niti.OP_RMSNORM_BWD, None, m, d))
    dgain = torch.empty(d, device="cuda")
    for extra in (None, dh):
        dx, intact = R.guarded(m, d, dtype, pad=1)
        niti.rmsnorm_bwd(dy, h, gain, rstd, dx, dgain, ws, dh=extra)
        want, bound, wg, mag = backward64(dy, h, gain, rstd, extra)
        R.close(dx, want, bound, dtype, "dx")
        intact()
        # a column's sum: rows of a workgroup in order (at most 5), partial rows of a group (at most 32), 16 groups
        R.close(dgain, wg, 64 * R.U32 * mag, what="dgain")
    again, dx2 = torch.empty_like(dgain), dh.clone()
    niti.rmsnorm_bwd(dy, h, gain, rstd, dx2, again, ws, dh=dx2)           # dx over dh, and the same sums again
    assert torch.equal(again, dgain) and torch.equal(dx2, dx)
    niti.rmsnorm_bwd(dy, h, gain, rstd, dx2)                              # no dgain, no workspace
    R.close(dx2, *backward64(dy, h, gain, rstd, None)[:2], dtype, "dx alone")


def test_backward_against_differences():
    """dx and dgain against central differences of the 64-bit forward pass."""
    m, d, eps = 3, 50, 1e-3
    x, dy = data(m, d, F32, 21), data(m, d, F32, 22)
    gain = 1 + 0.1 * data(1, d, F32, 23)[0]
    rstd, dx, dgain = torch.empty(m, device="cuda"), torch.empty_like(x), torch.empty(d, device="cuda")
    niti.rmsnorm_fwd(x, gain, rstd=rstd, eps=eps)
    niti.rmsnorm_bwd(dy, x, gain, rstd, dx, dgain, niti.new_workspace(niti.workspace_bytes(niti.OP_RMSNORM_BWD, None, m, d)))

    def loss(x64, g64):
        return (forward64(x64, None, g64, eps)[2] * dy.double().cpu()).sum()
    x64, g64, step = x.double().cpu(), gain.double().cpu(), 1e-5
    for i, j in ((0, 0), (1, 17), (2, 49), (1, 3)):
        e = torch.zeros(m, d, dtype=torch.float64)
        e[i, j] = step
        want = (loss(x64 + e, g64) - loss(x64 - e, g64)) / (2 * step)
        # third derivatives of order 10 times step^2, and the 64-bit sums' rounding over step
        assert abs(float(dx[i, j]) - float(want)) < 1e-5 * max(1, abs(float(want)))
        e = torch.zeros(d, dtype=torch.float64)
        e[j] = step
        want = (loss(x64, g64 + e) - loss(x64, g64 - e)) / (2 * step)
        assert abs(float(dgain[j]) - float(want)) < 1e-5 * max(1, abs(float(want)))


@pytest.mark.parametrize("mode", [niti.RTN, niti.SR])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("m,d", SHAPES)
def test_quantize(m, d, dtype, mode):
    say("quantize_rows", m, d, dtype, mode)
    x = data(m, d, dtype, 31, 0.02)
    x[0] = 0
    q, iq = R.guarded(m, d, torch.int8)
    y, iy = R.guarded(m, d, dtype)
    scale = torch.zeros(m, device="cuda")
    niti.quantize_rows(x, q, scale, y=y, mode=mode, seed=2 ** 63 + 5, call=3)
    x64 = x.double().cpu()
    s = R.scales(x64)
    R.close(scale, s, R.U32 * s, what="scale")
    u = R.field(R.draws(2 ** 63 + 5, 3, m * d), 40, 24).view(m, d) if mode == niti.SR else None
    R.check_codes(q, x64, s, u)
    R.close(y, q.double().cpu() * scale.double().cpu()[:, None], 0.0, dtype, "y")
    iq(), iy()


def test_stochastic_codes_are_right_on_average():
    x = torch.linspace(-1, 1, 4001, device="cuda").repeat(400, 1)
    q, scale = torch.empty(400, 4001, dtype=torch.int8, device="cuda"), torch.empty(400, device="cuda")
    niti.quantize_rows(x, q, scale, mode=niti.SR, seed=9)
    mean = (q.double() * scale.double()[:, None]).mean(dim=0)
    # a code's deviation is at most half a step: six of the mean's deviations
    assert (mean - x[0].double()).abs().max() < 6 * 0.5 / 127 / 400 ** 0.5


def test_quantize_special_rows():
    x = data(4, 77, F32, 41)
    x[0, 3], x[1, 5], x[2] = float("-inf"), float("nan"), 2.0 ** -120
    q, scale, y = torch.empty(4, 77, dtype=torch.int8, device="cuda"), torch.empty(4, device="cuda"), torch.empty_like(x)
    niti.quantize_rows(x, q, scale, y=y)
    assert (q[:3] == 0).all() and torch.isnan(scale[:2]).all() and torch.isnan(y[:2]).all()
    assert float(scale[2]) > 0 and (y[2] == 0).all() and int(q[3].abs().max()) == 127


def test_refusals():
    x, gain = torch.zeros(4, 8, device="cuda"), torch.ones(8, device="cuda")
    q, s = torch.zeros(4, 8, dtype=torch.int8, device="cuda"), torch.zeros(4, device="cuda")
    with pytest.raises(TypeError):
        niti.rmsnorm_fwd(x.cpu(), gain, y=x)
    with pytest.raises(TypeError):
        niti.rmsnorm_fwd(x.double(), gain, y=x)
    with pytest.raises(TypeError):
        niti.rmsnorm_fwd(x, gain, y=x.half())
    with pytest.raises(ValueError):
        niti.rmsnorm_fwd(x, gain[:7], y=x)
    with pytest.raises(ValueError):
        niti.rmsnorm_fwd(x.t(), torch.ones(4, device="cuda"), y=torch.zeros(8, 4, device="cuda"))
    with pytest.raises(ValueError):
        niti.rmsnorm_fwd(x, gain, y=x[:1].expand(4, 8))          # rows of an output overlap
    with pytest.raises(niti.NitiError):
        niti.rmsnorm_fwd(x, gain, q=q)                           # codes without scales
    with pytest.raises(niti.NitiError):
        niti.rmsnorm_fwd(x, gain, y=x, eps=-1.0)
    with pytest.raises(niti.NitiError):
        niti.quantize_rows(x, q, s, mode=niti.PSR)
    with pytest.raises(niti.NitiError):
        niti.rmsnorm_bwd(x, x, gain, s, x, gain.clone())         # dgain without a workspace
