"""Rows whose squares leave the normal range of 32 bits, below and above, with an
eps of their size or none."""
import pytest
import torch

import scaled_ref as R
from helpers import say
from paper_2009_13108_amd import niti
from test_gpu_rownorm import F32, Y_REL, data, forward64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("eps", [0.0, 1e-44, 1e-38, 1e-32, 1e-12, 1e36, 1e38])
@pytest.mark.parametrize("d", [5, 300, 1111, 4096, 9000, 20000, 40000])
def test_rows_of_any_size(d, eps):
    say("rmsnorm_fwd sizes", d, eps)
    sizes = [10.0 ** e for e in (-41, -37, -30, -24, -22, -20, -18, -16, -13, -3, 3, 18, 19, 20, 25, 37)]
    x = data(len(sizes), d, F32, 1).clamp(-3, 3) * torch.tensor(sizes, device="cuda")[:, None]
    gain = 1 + 0.1 * data(1, d, F32, 2)[0]
    eps = float(torch.tensor(eps, dtype=F32))
    _, rstd, want = forward64(x, None, gain, eps)
    y, got = torch.empty_like(x), torch.empty(len(sizes), device="cuda")
    q, scale = torch.empty(len(sizes), d, dtype=torch.int8, device="cuda"), torch.empty(len(sizes), device="cuda")
    niti.rmsnorm_fwd(x, gain, y=y, rstd=got, eps=eps)
    # a value below the normal range is off by the steps there: its own, and those of the factors before it
    R.close(y, want, Y_REL * want.abs() + 2.0 ** -148, what="y")
    held = rstd < 3e38
    R.close(got[held.cuda()], rstd[held], 25 * R.U32 * rstd[held] + 2.0 ** -148, what="rstd")
    assert torch.isinf(got[~held.cuda()]).all()
    niti.rmsnorm_fwd(x, gain, q=q, scale=scale, eps=eps)
    for i in range(len(sizes)):
        s = R.scales(want[i:i + 1])
        if float(s) > 2 * R.TINY / 127:
            R.check_codes(q[i:i + 1], want[i:i + 1], s, what="size %g" % sizes[i])
            R.close(scale[i:i + 1], s, 40 * R.U32 * s, what="scale")
