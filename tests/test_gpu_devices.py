"""Calls on tokens, logits and pairs of columns whose tensors or stream are not on the
current device are refused before anything is launched."""
import types

import pytest
import torch

from paper_2009_13108_amd import niti

pytestmark = pytest.mark.gpu


def calls():
    x, t = torch.zeros(2, 8, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    q, b, s, s8 = (torch.zeros(2, 8, dtype=torch.int8, device="cuda"), torch.zeros(16, 8, dtype=torch.int8, device="cuda"),
                   torch.ones(2, device="cuda"), torch.ones(16, device="cuda"))
    z, ws, idx = torch.zeros(2, 16, device="cuda"), niti.new_workspace(1 << 16), torch.zeros(2, 1, dtype=torch.int32, device="cuda")
    v = torch.zeros(2, 1, device="cuda")
    return [lambda **k: niti.gated_fwd(q, b, x, s, s8, **k), lambda **k: niti.gated_bwd(x, z, q, b, s, s8, ws, da=x.clone(), **k),
            lambda **k: niti.embedding_fwd(x, t, x.clone(), **k), lambda **k: niti.embedding_bwd(x, t, x.clone(), ws, **k),
            lambda **k: niti.token_logprobs(x, lse=s.clone(), **k), lambda **k: niti.distill_fwd(x, v, idx, s.clone(), **k),
            lambda **k: niti.distill_bwd(x, v, idx, s, None, x.clone(), **k)]


def test_another_current_device(monkeypatch):
    niti.token_logprobs(torch.zeros(1, 4, device="cuda"), lse=torch.zeros(1, device="cuda"))
    work = calls()
    for call in work:
        call()
        call(stream=torch.cuda.Stream())
    torch.cuda.synchronize()
    for call in work:
        with pytest.raises(ValueError, match="device"):
            call(stream=types.SimpleNamespace(device_index=1, cuda_stream=0))
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1)
    for call in work:
        with pytest.raises(ValueError, match="device"):
            call()
