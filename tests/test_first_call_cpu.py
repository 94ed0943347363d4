"""The binding's checks in the first call that a process makes, whichever it is."""
import pytest
import torch

from paper_2009_13108_amd import niti

X, T, Q, S, I = torch.zeros(2, 4), torch.zeros(2, dtype=torch.int32), torch.zeros(2, 4, dtype=torch.int8), torch.ones(2), torch.zeros(2, 1, dtype=torch.int32)
CALLS = {
    "rmsnorm_fwd": lambda: niti.rmsnorm_fwd(X, S), "rmsnorm_bwd": lambda: niti.rmsnorm_bwd(X, X, S, S, X),
    "quantize_rows": lambda: niti.quantize_rows(X, Q, S), "linear_fwd": lambda: niti.linear_fwd(Q, Q, X, S, S),
    "linear_bwd": lambda: niti.linear_bwd(X, Q, Q, S, S, None), "gated_fwd": lambda: niti.gated_fwd(Q, Q, X, S, S),
    "gated_bwd": lambda: niti.gated_bwd(X, X, Q, Q, S, S, None), "embedding_fwd": lambda: niti.embedding_fwd(X, T, X),
    "embedding_bwd": lambda: niti.embedding_bwd(X, T, X, None), "token_logprobs": lambda: niti.token_logprobs(X, lse=S),
    "distill_fwd": lambda: niti.distill_fwd(X, X, I, S), "distill_bwd": lambda: niti.distill_bwd(X, X, I, S, None, X),
    "adamw_plan": lambda: niti.adamw_plan([1], [1], [1], [1]),
}


@pytest.mark.parametrize("name", list(CALLS))
def test_first_call(name, monkeypatch):
    for state in ("_torch_mod", "_Tensor", "_raw_stream"):
        monkeypatch.setattr(niti, state, None)
    monkeypatch.setattr(niti, "_types", {})
    with pytest.raises(TypeError, match="must be .*device tensor"):
        CALLS[name]()
