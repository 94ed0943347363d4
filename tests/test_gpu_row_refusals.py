"""Operands that are missing or no tensors: the binding says which, as for any other
operand, before it marshals anything."""
import pytest
import torch

from paper_2009_13108_amd import niti

pytestmark = pytest.mark.gpu


def test_missing_operands():
    x, gain = torch.zeros(4, 16, device="cuda"), torch.ones(16, device="cuda")
    a, b = torch.zeros(4, 16, dtype=torch.int8, device="cuda"), torch.zeros(6, 16, dtype=torch.int8, device="cuda")
    out, s_a, s_b, rstd = torch.zeros(4, 6, device="cuda"), torch.ones(4, device="cuda"), torch.ones(6, device="cuda"), torch.ones(4, device="cuda")
    for bad in (None, 3.0, [1, 2]):
        for call, what in ((lambda: niti.rmsnorm_fwd(x, bad, y=x), "gain"), (lambda: niti.rmsnorm_fwd(bad, gain, y=x), "x"),
                           (lambda: niti.rmsnorm_bwd(x, x, bad, rstd, x), "gain"), (lambda: niti.linear_fwd(a, bad, out, s_a, s_b), "b"),
                           (lambda: niti.linear_fwd(a, b, bad, s_a, s_b), "out"), (lambda: niti.linear_fwd(a, b, out, bad, s_b), "s_a"),
                           (lambda: niti.linear_bwd(out, bad, b, s_a, s_b, None), "a"), (lambda: niti.quantize_rows(bad, a, s_a), "x")):
            with pytest.raises(TypeError, match="^%s must be a device tensor" % what):
                call()
    with pytest.raises(ValueError, match="b must be a matrix"):
        niti.linear_fwd(a, b[0], out, s_a, s_b)
    with pytest.raises(TypeError, match="x must be a device tensor"):
        niti.rmsnorm_fwd(x.cpu(), gain, y=x)


def test_plans_of_what_is_no_tensor():
    p = torch.zeros(8, device="cuda")
    for i, what in enumerate(("params", "grads", "m", "v")):
        args = [[p], [p], [p.clone()], [p.clone()]]
        args[i] = [None]
        with pytest.raises(TypeError, match="%s must be device tensors" % what):
            niti.adamw_plan(*args)
