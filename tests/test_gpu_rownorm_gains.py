"""Norm and its gradients with gains of every type: the matrix's own, 32 bits beside
16, and the other 16-bit type, which the kernels for rows of any length take."""
import pytest
import torch

import scaled_ref as R
from helpers import say
from paper_2009_13108_amd import niti
from test_gpu_rownorm import BF16, F16, F32, SHAPES, Y_REL, backward64, data, forward64

pytestmark = pytest.mark.gpu
TYPES = [F32, BF16, F16]


@pytest.mark.parametrize("gain_type", TYPES)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,d", SHAPES + [(70, 1000), (5, 16384), (3, 20000)])
def test_forward(m, d, dtype, gain_type):
    say("rmsnorm_fwd gain", m, d, dtype, gain_type)
    x, res = data(m, d, dtype, 1), data(m, d, dtype, 2)
    gain = (1 + 0.1 * data(1, d, F32, 3)[0]).to(gain_type)
    h64, rstd64, y64 = forward64(x, res, gain, 1e-5)
    (h, ih), (y, iy), (q, iq) = R.guarded(m, d, dtype), R.guarded(m, d, dtype, pad=3), R.guarded(m, d, torch.int8, pad=5)
    scale, rstd = torch.zeros(m, device="cuda"), torch.zeros(m, device="cuda")
    niti.rmsnorm_fwd(x, gain, res=res, h=h, y=y, q=q, scale=scale, rstd=rstd, eps=1e-5)
    R.close(h, h64, R.U32 * h64.abs(), dtype, "h")
    R.close(rstd, rstd64, 25 * R.U32 * rstd64, what="rstd")
    s = R.scales(y64)
    R.close(scale, s, (Y_REL + 2 * R.U32) * s, what="scale")
    R.check_codes(q, y64, s)
    R.close(y, q.double().cpu() * scale.double().cpu()[:, None], R.U32 * (127 * scale.double().cpu()[:, None]), dtype, "y of codes")
    niti.rmsnorm_fwd(x, gain, res=res, y=y, eps=1e-5)
    R.close(y, y64, Y_REL * y64.abs(), dtype, "y")
    ih(), iy(), iq()


@pytest.mark.parametrize("gain_type", TYPES)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,d", SHAPES + [(2100, 96), (1030, 2500), (515, 9000), (17, 1000), (5, 4096)])
def test_backward(m, d, dtype, gain_type):
    say("rmsnorm_bwd gain", m, d, dtype, gain_type)
    h, dy, dh = data(m, d, dtype, 11), data(m, d, dtype, 12, 0.1), data(m, d, dtype, 13, 0.1)
    gain = (1 + 0.1 * data(1, d, F32, 14)[0]).to(gain_type)
    rstd = (1 / torch.sqrt(h.double().square().mean(dim=1) + 1e-6)).float()
    ws = niti.new_workspace(niti.workspace_bytes(niti.OP_RMSNORM_BWD, None, m, d))
    dgain = torch.empty(d, device="cuda")
    for extra in (None, dh):
        dx, intact = R.guarded(m, d, dtype, pad=1)
        niti.rmsnorm_bwd(dy, h, gain, rstd, dx, dgain, ws, dh=extra)
        want, bound, wg, mag = backward64(dy, h, gain, rstd, extra)
        R.close(dx, want, bound, dtype, "dx")
        # a column's sum: a workgroup's rows in order (16 at most where it is the only one, 1 + M / 512 or 1 + M / 2048 else),
        # 16 partial rows of each of 32 groups, and three and seven joins of those
        R.close(dgain, wg, 64 * R.U32 * mag, what="dgain")
        intact()
