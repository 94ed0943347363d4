"""Calls on tokens, logits and pairs of columns on another stream than the current one, ordered by events, each with
a workspace of its own: the same results as on the current stream."""
import pytest
import torch

from paper_2009_13108_amd import niti
from test_gpu_logits import F32, logits, some_tokens, teacher_of

pytestmark = pytest.mark.gpu


def calls():
    """(the call on given outputs and workspace, its outputs' shapes, its workspace's size)"""
    m, f, k, v, d = 70, 96, 80, 140000, 50
    g = torch.Generator(device="cuda").manual_seed(1)
    codes = lambda r, c: torch.randint(-127, 128, (r, c), generator=g, device="cuda", dtype=torch.int8)  # noqa: E731
    rand = lambda *s: torch.rand(s, generator=g, device="cuda") + 0.1  # noqa: E731
    a, b, sa, sb, dy, z, table = codes(m, k), codes(2 * f, k), rand(m), rand(2 * f), rand(m, f), rand(m, 2 * f), rand(300, d)
    tok, dout, x, at = some_tokens(m, 300, 2), rand(m, d), logits(3, v, F32, 3), some_tokens(3, v, 4)
    tv, ti = teacher_of(x, 8, 5, F32)
    lse = torch.logsumexp(x, dim=1)
    need = niti.workspace_bytes
    return [
        (lambda o, ws, s: niti.gated_fwd(a, b, o[0], sa, sb, z=o[1], ws=ws, stream=s), [(m, f), (m, 2 * f)], need(niti.OP_GATED_FWD, None, m, f, k)),
        (lambda o, ws, s: niti.gated_bwd(dy, z, a, b, sa, sb, ws, da=o[0], db=o[1], dbias=o[2], stream=s), [(m, k), (2 * f, k), (2 * f,)],
         need(niti.OP_GATED_BWD, None, m, f, k)),
        (lambda o, ws, s: niti.embedding_fwd(table, tok, o[0], stream=s), [(m, d)], 0),
        (lambda o, ws, s: niti.embedding_bwd(dout, tok, o[0], ws, stream=s), [(300, d)], need(niti.OP_EMBEDDING_BWD, None, m, 300, d)),
        (lambda o, ws, s: niti.token_logprobs(x, tokens=at, logp=o[0], lse=o[1], entropy=o[2], ws=ws, stream=s), [(3,)] * 3,
         need(niti.OP_TOKEN_LOGPROBS, None, 3, v, 0)),
        (lambda o, ws, s: niti.distill_fwd(x, tv, ti, o[0], lse=o[1], dlogits=o[2], ws=ws, stream=s), [(3,), (3,), (3, v)],
         need(niti.OP_DISTILL_FWD, None, 3, v)),
        (lambda o, ws, s: niti.distill_bwd(x, tv, ti, lse, None, o[0], stream=s), [(3, v)], 0),
    ]


def test_another_stream():
    work = calls()
    sides = [torch.cuda.Stream() for _ in work]
    outs = [[[torch.full(s, 7.0, device="cuda") for s in shapes] for _ in range(2)] for _, shapes, _ in work]
    spaces = [[niti.new_workspace(n) for _ in range(2)] for _, _, n in work]
    for side in sides:
        side.wait_stream(torch.cuda.current_stream())
    # all of them at once, and on the current stream meanwhile
    for (call, _, _), side, out, ws in zip(work, sides, outs, spaces):
        call(out[0], ws[0], side)
        call(out[1], ws[1], None)
    for side in sides:
        torch.cuda.current_stream().wait_stream(side)
    for i, (a, b) in enumerate(outs):
        for s, t in zip(a, b):
            assert torch.equal(s, t) and not (t == 7.0).all(), i
