"""Activations and their slopes in 32 bits against their 64-bit forms, over all z
that matter and on their own: a product of nothing leaves the bias as z, and with
one row dbias is the slope.  U is one rounding's relative error, 2^-24."""
import math

import pytest
import torch

from helpers import say
from paper_2009_13108_amd import niti
from scaled_ref import U32 as U

pytestmark = pytest.mark.gpu
N = 1 << 21


def grid(lo, hi, seed):
    """z between lo and hi: evenly spread, and their magnitudes' logarithms too."""
    g = torch.Generator().manual_seed(seed)
    even = lo + (hi - lo) * torch.rand(N // 2, generator=g, dtype=torch.float64)
    small = (hi if hi > 0 else lo) * torch.exp(-20 * torch.rand(N // 2, generator=g, dtype=torch.float64))
    return torch.cat([even, small]).float().cuda()


def value(z, act):
    a, b = torch.zeros(1, 0, dtype=torch.int8, device="cuda"), torch.zeros(z.numel(), 0, dtype=torch.int8, device="cuda")
    out, one = torch.empty(1, z.numel(), device="cuda"), torch.ones(1, device="cuda")
    niti.linear_fwd(a, b, out, one, one, bias=z, act=act)
    return out[0].double()


def slope(z, act):
    n = z.numel()
    a, b = torch.zeros(1, 1, dtype=torch.int8, device="cuda"), torch.zeros(n, 1, dtype=torch.int8, device="cuda")
    dbias, one = torch.empty(n, device="cuda"), torch.ones(1, device="cuda")
    most = min(n, 1 << 16)   # columns of one call
    ws = niti.new_workspace(niti.workspace_bytes(niti.OP_LINEAR_BWD, None, 1, most, 1))
    for at in range(0, n, most):
        part = z[at:at + most].view(1, -1)
        k = part.shape[1]
        niti.linear_bwd(torch.ones_like(part), a, b[:k], one, one, ws, z=part, act=act, dbias=dbias[at:at + k])
    return dbias.double()


def gelu_bounds(z):
    """Bounds of the distribution function's error, in U.  Its tail q = e Q(t): t is off by 3 U, which Q passes
    on at most once, Q by 2 and its fit, the product by 1, e by 2 and three roundings of its exponent z^2 / 2;
    below |z| = 1.25, 1/2 + z P(z^2) is off by 0.8 and its own rounding."""
    q = torch.special.erfc(z.abs() / math.sqrt(2)) / 2
    tail = q * (9 + 1.5 * z * z)
    return torch.where(z < 0, torch.where(z.abs() < 1.25, q + 0.8, tail), 1.8 + tail)


@pytest.mark.parametrize("lo,hi", [(-12.4, 0.0), (0.0, 12.4), (-1.3, 1.3)])
def test_gelu(lo, hi):
    say("gelu", lo, hi)
    z = grid(lo, hi, 1)
    z64 = z.double()
    want = z64 * torch.special.erfc(-z64 / math.sqrt(2)) / 2
    bound = U * (z64.abs() * gelu_bounds(z64) + want.abs()) * 1.01 + 2.0 ** -140
    off = (value(z, niti.ACT_GELU) - want).abs()
    assert (off <= bound).all(), (float(z[(off / bound).argmax()]), float((off / bound).max()))


@pytest.mark.parametrize("lo,hi", [(-12.4, 0.0), (0.0, 12.4), (-1.3, 1.3)])
def test_gelu_slope(lo, hi):
    say("gelu slope", lo, hi)
    z = grid(lo, hi, 2)
    z64 = z.double()
    density = z64 * torch.exp(-z64 * z64 / 2) / math.sqrt(2 * math.pi)
    want = torch.special.erfc(-z64 / math.sqrt(2)) / 2 + density
    bound = U * (gelu_bounds(z64) + density.abs() * (5 + 1.5 * z64 * z64) + want.abs()) * 1.01 + 2.0 ** -140
    off = (slope(z, niti.ACT_GELU) - want).abs()
    assert (off <= bound).all(), (float(z[(off / bound).argmax()]), float((off / bound).max()))


@pytest.mark.parametrize("lo,hi", [(-79.0, 0.0), (0.0, 79.0), (-3.0, 3.0)])
def test_silu(lo, hi):
    """s = 1 / (1 + e), e = exp(-z): e is off by 2 and two roundings of its exponent, the sum by 1, the reciprocal by 2."""
    say("silu", lo, hi)
    z = grid(lo, hi, 3)
    z64 = z.double()
    s = torch.sigmoid(z64)
    rel = (1 - s) * (2 * z64.abs() + 2) + 4
    want = z64 * s
    off = (value(z, niti.ACT_SILU) - want).abs()
    bound = U * want.abs() * rel * 1.01 + 2.0 ** -140
    assert (off <= bound).all(), (float(z[(off / bound).argmax()]), float((off / bound).max()))


def test_relu_and_ends():
    z = torch.tensor([-3.0, -0.0, 0.0, 2.5, float("inf"), float("-inf"), float("nan"), 3e38, -3e38], device="cuda")
    assert torch.equal(value(z, niti.ACT_RELU)[:5], torch.tensor([0, 0, 0, 2.5, float("inf")], device="cuda").double())
    for act in (niti.ACT_GELU, niti.ACT_SILU):
        v = value(z, act)
        assert float(v[4]) == float("inf") and abs(float(v[5])) < 1e-30 and torch.isnan(v[6])
        assert float(v[7]) == float(z[7]) and abs(float(v[8])) < 1e-30
        d = slope(z, act)
        assert torch.equal(d[[4, 7]], torch.ones(2, dtype=torch.float64, device="cuda")) and (d[[5, 8]].abs() < 1e-30).all()
        assert torch.isnan(d[6])
