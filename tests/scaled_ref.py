"""64-bit forms of the operators on int8 rows, written from their formulas,
and the error bounds that their 32-bit evaluation allows.

U32 = 2^-24 is the relative error of one rounding to 32 bits; UNIT[dtype] that
of the one rounding at a store.  A 32-bit sum of n terms in a tree of depth k
is off by at most k U32 times the sum of the magnitudes; the kernels' sums per
row have at most 32 terms a thread and 10 tree levels."""
import math

import numpy as np
import torch

U32 = 2.0 ** -24
UNIT = {t: torch.finfo(t).eps / 2 for t in (torch.float32, torch.bfloat16, torch.float16)}   # half a step at 1: 2^-24, 2^-8, 2^-11
# the smallest step of a type (below its normal range a rounding is off by half of it)
STEP = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}
TINY = 2.0 ** -100
# A value formed in 32 bits and divided by its row's scale: at most 127, each of
# rstd (sum, root, division), the products and the scale off by less than 50 U32
# in all, so a code's argument is off by less than 127 * 100 U32 < 0.001.
CODE_SLACK = 0.001


def close(got, want, bound, dtype=torch.float32, what=""):
    """|got - want| <= bound + one rounding to dtype; NaNs and infinities in the same places."""
    got, want = got.double().cpu(), want.double().cpu()
    assert got.shape == want.shape, what
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what + ": NaNs differ"
    fine = torch.isfinite(want)
    assert torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)]), what
    # the value before the store is x with |x - want| <= bound, and its rounding is off by UNIT |x| <= UNIT (|want| + bound)
    bound = torch.as_tensor(bound, dtype=torch.float64).cpu()
    room = (bound + UNIT[dtype] * (want.abs() + bound) * 1.01 + STEP[dtype]).expand(want.shape)
    off = (got - want).abs()
    bad = (off > room) & fine
    assert not bad.any(), "%s: %d of %d off, by up to %g (allowed there %g)" % (
        what, int(bad.sum()), bad.numel(), float(off[bad].max()), float(room[bad][off[bad].argmax()]))


def draws(seed, call, n):
    """SplitMix64 outputs call 2^40 + 1 .. call 2^40 + n."""
    u = np.uint64
    with np.errstate(over="ignore"):
        z = u(seed) + (u((call << 40) & (2 ** 64 - 1)) + np.arange(1, n + 1, dtype=u)) * u(0x9E3779B97F4A7C15)
        z ^= z >> u(30)
        z *= u(0xBF58476D1CE4E5B9)
        z ^= z >> u(27)
        z *= u(0x94D049BB133111EB)
        z ^= z >> u(31)
    return z


def field(z, low, bits):
    return torch.from_numpy(((z >> np.uint64(low)) & np.uint64((1 << bits) - 1)).astype(np.float64) / 2.0 ** bits)


def scales(x, dim=1):
    top = x.abs().amax(dim=dim) if x.numel() else torch.zeros(x.shape[1 - dim], dtype=x.dtype)
    return top.clamp(min=TINY) / 127


def check_codes(q, x, scale64, u=None, what="codes"):
    """Codes q of x (64 bits): rint(x / scale) or floor(x / scale + u), where the argument may be off by CODE_SLACK."""
    r = x / scale64[:, None]
    q = q.double().cpu()
    assert q.abs().max() <= 127 if q.numel() else True
    if u is None:
        off = (q - r).abs() - 0.5
    else:   # floor(r + u): q <= r + u < q + 1, held to 127
        off = torch.maximum(q - (r + u), torch.where(q < 127, (r + u) - (q + 1), torch.full_like(q, -1.0)))
    assert (off <= CODE_SLACK).all(), "%s: off by %g" % (what, float(off.max()))


def act(name, z):
    if name == "relu":
        return z.clamp(min=0)
    if name == "gelu":
        return 0.5 * z * torch.erfc(-z / math.sqrt(2))
    if name == "silu":
        return z * torch.sigmoid(z)
    return z


def slope(name, z):
    if name == "relu":
        return (z > 0).double()
    if name == "gelu":
        return 0.5 * torch.erfc(-z / math.sqrt(2)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if name == "silu":
        s = torch.sigmoid(z)
        return s + z * s * (1 - s)
    return torch.ones_like(z)


def guarded(rows, cols, dtype, pad=0, fill=77):
    """A matrix inside a larger one, and a check that nothing around it was written."""
    big = torch.full((rows + 2, cols + pad + 16), fill, dtype=dtype, device="cuda")
    view = big[1:rows + 1, 8:8 + cols]
    before = big.clone()

    def intact():
        after = big.clone()
        after[1:rows + 1, 8:8 + cols] = before[1:rows + 1, 8:8 + cols]
        assert torch.equal(after, before), "written outside the output"
    return view, intact
