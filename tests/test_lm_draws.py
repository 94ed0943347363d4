"""Stochastic draws of the token model: no two calls of its training share any.  The
library's calls are stand-ins here that note their seeds and indices."""
import types

import torch

from paper_2009_13108_amd import lm, niti


def test_no_draw_is_used_twice(monkeypatch):
    used = []

    def note(mode, seed, call):
        if mode == niti.SR:
            used.append((seed & 0xFFFFFFFFFFFFFFFF, call & 0xFFFFFFFF))

    def gradients(*args, mode=niti.RTN, seed=0, call=0, **kw):
        note(mode, seed, call)

    def adamw_plan(params, grads, m, v, m_scale=None, v_scale=None):
        return types.SimpleNamespace(bits=32 if m_scale is None else 8)

    def adamw_step(plan, step, lr, mode=niti.RTN, seed=0, **kw):
        if plan.bits == 8:      # draws of call = step
            note(mode, seed, step)

    nothing = lambda *args, **kw: None  # noqa: E731
    calls = dict.fromkeys(("embedding_fwd", "embedding_bwd", "rmsnorm_fwd", "rmsnorm_bwd", "gated_fwd", "linear_fwd", "distill_fwd"), nothing)
    calls.update(quantize_rows=gradients, linear_bwd=gradients, gated_bwd=gradients, adamw_plan=adamw_plan, adamw_step=adamw_step,
                 workspace_bytes=lambda *a: 0)
    for name, f in calls.items():
        monkeypatch.setattr(niti, name, f)
    for seed in (0, 1, 7, 2 ** 63 - 1):
        del used[:]
        net = lm.TokenModel(8, 4, 4, 2, torch.float32, 2, state_bits=8, mode=niti.SR, seed=seed, device="cpu")
        for _ in range(300):
            net.forward(None)
            net.teach(None, None, None)
            net.step()
        assert len(used) == 4 * 300 == len(set(used))
