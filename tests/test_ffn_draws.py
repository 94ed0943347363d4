"""Stochastic draws of the feed-forward block: no two calls of its training share
any.  The library's calls are stand-ins here that note their seeds and indices."""
import types

import torch

from paper_2009_13108_amd import ffn, niti


def test_no_draw_is_used_twice(monkeypatch):
    used = []

    def note(seed, call):
        used.append((seed & 0xFFFFFFFFFFFFFFFF, call & 0xFFFFFFFF))

    def quantize_rows(x, q, scale, y=None, mode=niti.RTN, seed=0, call=0, stream=None):
        if mode == niti.SR:
            note(seed, call)

    def linear_bwd(*args, mode=niti.RTN, seed=0, call=0, **kw):
        if mode == niti.SR:
            note(seed, call)

    def adamw_plan(params, grads, m, v, m_scale=None, v_scale=None):
        return types.SimpleNamespace(bits=32 if m_scale is None else 8)

    def adamw_step(plan, step, lr, mode=niti.RTN, seed=0, **kw):
        if plan.bits == 8 and mode == niti.SR:      # draws of call = step
            note(seed, step)

    nothing = lambda *args, **kw: None  # noqa: E731
    for name, f in dict(quantize_rows=quantize_rows, linear_bwd=linear_bwd, adamw_plan=adamw_plan, adamw_step=adamw_step,
                        linear_fwd=nothing, rmsnorm_fwd=nothing, rmsnorm_bwd=nothing, workspace_bytes=lambda *a: 0).items():
        monkeypatch.setattr(niti, name, f)
    for seed in (0, 1, 7, 2 ** 63 - 1):
        del used[:]
        net = ffn.FeedForward(8, 16, 4, torch.float32, seed=seed, device="cpu")
        x = torch.zeros(4, 8)
        for _ in range(20):
            net.forward(x)
            net.backward(x)
            net.step()
        assert len(used) == 60 and len(set(used)) == 60, (seed, sorted(used)[:6])
