"""AdamW where the second moment, or eps, lies below the normal range of 32 bits."""
import math

import pytest
import torch

import scaled_ref as R
from helpers import say
from paper_2009_13108_amd import niti

pytestmark = pytest.mark.gpu
LR, B1, B2 = 1e-2, 0.9, 0.999


@pytest.mark.parametrize("eps", [0.0, 1e-42, 1e-30, 1e-20, 1e-8])
@pytest.mark.parametrize("step", [1, 7, 5000])
def test_small_gradients(step, eps):
    """Parameters from the step's own m and v, in 64 bits: the divisor's root, its correction, sum and reciprocal
    and the products after it are 12 roundings at most, the rate's own among them."""
    say("adamw small", step, eps)
    n = 4096
    g = (10.0 ** torch.linspace(-24, -3, n, dtype=torch.float64)).float().cuda()
    g[1::2].neg_()
    p = torch.zeros(n, device="cuda")
    m, v = g * 0.3, (g * g) * 0.5
    niti.adamw_step(niti.adamw_plan([p], [g], [m], [v]), step, LR, beta1=B1, beta2=B2, eps=eps)
    m64, v64 = m.double().cpu(), v.double().cpu()
    up = LR / (1 - B1 ** step) * m64 / (torch.sqrt(v64 / (1 - B2 ** step)) + float(torch.tensor(eps, dtype=torch.float32)))
    assert int((v64 == 0).sum()) > 0 and int(((v64 > 0) & (v64 < 2.0 ** -126)).sum()) > 0
    R.close(p, -up, 12 * R.U32 * up.abs(), what="p")


def test_first_step_is_the_rate():
    """With eps = 0 the first step moves every parameter by the rate, whatever its gradient's size."""
    g = torch.tensor([1e-3, -1e-15, 1e-18, -1e-19, 3e-18, 1e-12], device="cuda")
    p = torch.zeros(6, device="cuda")
    m, v = torch.zeros_like(p), torch.zeros_like(p)
    niti.adamw_step(niti.adamw_plan([p], [g], [m], [v]), 1, LR, beta1=B1, beta2=B2, eps=0.0)
    # (v of 1e-19 is 1e-41, a multiple of 2^-149: 7e-5 from its value, and its root half of that)
    assert torch.allclose(p.cpu(), -LR * g.sign().cpu(), rtol=1e-4, atol=0)


def test_eight_bit_states_with_small_gradients():
    """Blocks above the least scale, 2^-100, with eps = 0: finite, and as large a step as the formula's."""
    n = 512
    g = torch.full((n,), 4e-15, device="cuda")
    g[256:] = 1e-3
    p, m, v = torch.zeros(n, device="cuda"), torch.zeros(n, dtype=torch.int8, device="cuda"), torch.zeros(n, dtype=torch.uint8, device="cuda")
    sm, sv = torch.zeros(2, device="cuda"), torch.zeros(2, device="cuda")
    niti.adamw_step(niti.adamw_plan([p], [g], [m], [v], [sm], [sv]), 1, LR, beta1=B1, beta2=B2, eps=0.0)
    assert math.isfinite(float(p.sum())) and torch.allclose(p, torch.full_like(p, -LR), rtol=1e-5, atol=0)


@pytest.mark.parametrize("step,limit", [(1, 2.0 ** -36 / math.sqrt(1 - B2)), (100000, 2.0 ** -36)])
@pytest.mark.parametrize("factor", [0.98, 1.02])
def test_both_sides_of_the_least_plain_eps(step, limit, factor):
    """eps just below and above what lets the hardware's roots be taken as they are."""
    test_small_gradients(step, limit * factor)
