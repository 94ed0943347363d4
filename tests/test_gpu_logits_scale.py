"""The ends of the scale of logits: factors whose product with log2 e is no number are refused, the largest
ones that are not, and the smallest, give numbers."""
import ctypes
import math

import pytest
import torch

from paper_2009_13108_amd import niti

FAKE = ctypes.c_void_p(0x100000)   # never dereferenced: every call on it fails validation
LARGEST = 2.0 ** 127


@pytest.mark.parametrize("scale", [LARGEST * (1 + 2 ** -20), 2.4e38, 3.4e38])
def test_larger_scales_are_refused(scale):
    lib = niti.lib()
    assert lib.niti_token_logprobs(FAKE, 40, None, None, FAKE, None, None, None, 3, 40, 0, scale, 0, None, 0, None) == -6
    assert lib.niti_distill_fwd(FAKE, 40, FAKE, 4, 0, FAKE, 4, FAKE, None, None, 0, None, 0, 3, 40, 4, scale, 0, None, 0, None) == -6
    assert lib.niti_distill_bwd(FAKE, 40, FAKE, 4, 0, FAKE, 4, FAKE, None, 0, FAKE, 40, 3, 40, 4, scale, 0, None) == -6


@pytest.mark.gpu
@pytest.mark.parametrize("v", [6, 64, 5000, 40000, 70000])
@pytest.mark.parametrize("base", [0.0, 0.5, -2.0 ** -120])
def test_largest_scale(v, base):
    """Any logit below the row's largest has no share: four equals have a quarter each."""
    x = torch.full((2, v), base - 1.0, device="cuda")
    x[1] = -torch.inf
    top = torch.tensor([0, 2, v // 2, v - 1], device="cuda") if v > 6 else torch.tensor([0, 2, 4, 5], device="cuda")
    x[:, top] = base
    rows = lambda *s, t=torch.float32: torch.full((2, *s), 7, dtype=t, device="cuda")  # noqa: E731
    ws = niti.new_workspace(max(niti.workspace_bytes(niti.OP_TOKEN_LOGPROBS, None, 2, v, 5), niti.workspace_bytes(niti.OP_DISTILL_FWD, None, 2, v)))
    logp, lse, entropy, top_logp, top_idx = rows(), rows(), rows(), rows(5), rows(5, t=torch.int32)
    tokens = torch.tensor([v - 1, 0], dtype=torch.int32, device="cuda")
    niti.token_logprobs(x, tokens=tokens, logp=logp, lse=lse, entropy=entropy, top_logp=top_logp, top_idx=top_idx, scale=LARGEST, ws=ws)
    # the logarithm of 4 by the library's function and its rounding, the product with scale exact
    four, off = math.log(4), 4 * 2.0 ** -24 * math.log(4)
    assert (logp.double() + four).abs().max() <= off and (entropy.double() - four).abs().max() <= off
    assert (top_logp[:, :4].double() + four).abs().max() <= off and (top_idx[:, :4] == top.int()).all()
    # (what is 1 below the maximum is 2^127 below it here)
    assert top_logp[0, 4] == -LARGEST and top_logp[1, 4] == -torch.inf
    want = LARGEST * base + four
    assert (lse.double() - want).abs().max() <= off + 2.0 ** -23 * abs(want)
    # a teacher that has two of them, and one that the student rules out at no probability
    t_val = torch.tensor([[3.0, 3.0, 1.0]], device="cuda").expand(2, 3).contiguous()
    t_idx = torch.stack([top[1], top[3], torch.tensor(1, device="cuda")]).to(torch.int32).expand(2, 3).contiguous()
    loss, dx, dx2 = rows(), rows(v), rows(v)
    dloss = torch.full((1,), 2.0 ** -100, device="cuda")
    niti.distill_fwd(x, t_val, t_idx, loss, lse=lse, dlogits=dx, dloss=dloss, scale=LARGEST, ws=ws)
    assert (loss.double() - math.log(2)).abs().max() <= 3 * off
    share = torch.zeros(v, dtype=torch.float64, device="cuda")
    share[top] = 0.25
    share[t_idx[0, :2].long()] -= 0.5
    assert (dx.double() - 2.0 ** 27 * share).abs().max() <= 2.0 ** 27 * 16 * 2.0 ** -24
    if base == 0.0:          # (what else lse is, it has no digits for the logarithm's)
        niti.distill_bwd(x, t_val, t_idx, lse, dloss, dx2, scale=LARGEST)
        assert (dx2.double() - 2.0 ** 27 * share).abs().max() <= 2.0 ** 27 * 16 * 2.0 ** -24


@pytest.mark.gpu
@pytest.mark.parametrize("v", [64, 5000, 70000])
def test_smallest_scale(v):
    """Every logit has the same share."""
    x = torch.randn(2, v, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    ws = niti.new_workspace(niti.workspace_bytes(niti.OP_TOKEN_LOGPROBS, None, 2, v, 0))
    lse, entropy = torch.zeros(2, device="cuda"), torch.zeros(2, device="cuda")
    for scale in (2.0 ** -149, 2.0 ** -126):
        niti.token_logprobs(x, lse=lse, entropy=entropy, scale=scale, ws=ws)
        # the sum is off by less than 156 roundings, its logarithm by two
        off = 2.0 ** -24 * (156 + 2 * math.log(v))
        assert (lse.double() - math.log(v)).abs().max() <= off and (entropy.double() - math.log(v)).abs().max() <= off
