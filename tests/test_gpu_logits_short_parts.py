"""Top alternatives where a row's last part has fewer columns than alternatives are asked for, and masks
there; and rows with fewer numbers than that.  Every place of the outputs is written, from this call's logits."""
import pytest
import torch

from helpers import say
from paper_2009_13108_amd import niti
from test_gpu_logits import BF16, F16, F32, NINF, check_logprobs, logits, run_logprobs, some_tokens

pytestmark = pytest.mark.gpu

# rows, the last part's first column: few rows in parts of 4096 columns, more in 8192 (32 bits) or 16384 (16 bits)
PLANS = [(6, 65536, F32), (6, 65536, BF16), (6, 65536, F16), (6, 98304, F32), (6, 98304, BF16), (102, 65536, F32), (54, 65536, BF16),
         (54, 65536, F16), (518, 16384, F32), (258, 32768, BF16)]


@pytest.mark.parametrize("last", [1, 5, 63])
@pytest.mark.parametrize("m,first,dtype", PLANS)
def test_masked_last_part(m, first, dtype, last):
    v = first + last
    say("short last part", m, v, dtype)
    x, tok = logits(m, v, dtype, 1), some_tokens(m, v, 2)
    x[1::6, first:] = NINF                    # the part is masked, the rest is not
    x[2::6, first + last // 2:] = NINF        # half of it
    x[3::6, : v - 3] = NINF                   # three columns at the end are all that is left
    x[4::6] = NINF
    x[4::6, 7] = 1.5
    x[5::6] = NINF
    for top in (1, 20, 64):
        check_logprobs(x, tok, top, 1.0)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_contents_of_the_workspace(dtype):
    """Whatever the workspace holds, a call gives the same again."""
    v = 65536 + 9
    x, tok = logits(3, v, dtype, 3), some_tokens(3, v, 4)
    x[0, 65536:] = NINF
    x[1, 65537:] = NINF
    first = run_logprobs(x, tok, 20, 1.0)
    for fill in (0, 0x3F, 0x7F, 0xFF):
        ws = niti.new_workspace(niti.workspace_bytes(niti.OP_TOKEN_LOGPROBS, None, 3, v, 20)).fill_(fill)
        out = {k: torch.full_like(t, 7) for k, t in first.items()}
        niti.token_logprobs(x, tokens=tok, ws=ws, **out)
        assert all(torch.equal(out[k], first[k]) for k in out), fill


@pytest.mark.parametrize("v", [5, 50, 9000, 40000, 65537, 140000])
def test_rows_of_few_numbers(v):
    """A NaN makes a row's outputs NaN and its columns -1, all of them, however few of the others are numbers."""
    top = min(20, v)
    x = torch.full((4, v), float("nan"), device="cuda")
    x[0, 1:4] = NINF
    x[1, 1], x[1, 2], x[1, 3] = NINF, 2.0, -1.0
    x[2], x[2, 0] = NINF, float("nan")
    x[3], x[3, v - 1] = NINF, float("inf")
    out = run_logprobs(x, some_tokens(4, v, 5), top, 1.0)
    for k in ("logp", "lse", "entropy", "top_logp"):
        assert torch.isnan(out[k]).all(), k
    assert (out["top_idx"] == -1).all()
