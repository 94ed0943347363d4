"""Operators on tokens and logits and the gated product: argument checks on the
host, before anything is launched."""
import ctypes

import pytest
import torch

from paper_2009_13108_amd import niti

FAKE = ctypes.c_void_p(0x100000)   # never dereferenced: every call below fails validation
ODD = ctypes.c_void_p(0x100008)
NULL = None
INF, NAN = float("inf"), float("nan")


def gated_fwd(a=FAKE, lda=16, sa=FAKE, san=4, b=FAKE, ldb=16, sb=FAKE, sbn=12, bias=NULL, bt=0, act=3, z=NULL, ldz=0, out=FAKE, ldout=6,
              M=4, F=6, K=16, type=0, ws=NULL, n=0):
    return niti.lib().niti_gated_fwd(a, lda, sa, san, b, ldb, sb, sbn, bias, bt, act, z, ldz, out, ldout, M, F, K, type, ws, n, None)


def test_gated_forward_rejects():
    assert gated_fwd(M=-1) == -2 and gated_fwd(F=-1) == -2 and gated_fwd(K=-1) == -2
    assert gated_fwd(type=3) == -6 and gated_fwd(act=4) == -6 and gated_fwd(act=-1) == -6 and gated_fwd(bias=FAKE, bt=7) == -6
    assert gated_fwd(K=1 << 17, lda=1 << 17, ldb=1 << 17) == -3 and gated_fwd(F=1 << 21) == -3 and gated_fwd(M=1 << 31) == -3
    for name in ("a", "b", "out", "sa", "sb"):
        assert gated_fwd(**{name: NULL}) == -1, name
    assert gated_fwd(san=3) == -2 and gated_fwd(sbn=6) == -2 and gated_fwd(lda=15) == -2 and gated_fwd(ldb=8) == -2
    assert gated_fwd(ldout=5) == -2 and gated_fwd(z=FAKE, ldz=6) == -2 and gated_fwd(n=64) == -4
    assert gated_fwd(M=0, a=NULL) == 0 and gated_fwd(F=0, out=NULL) == 0


def gated_bwd(dy=FAKE, lddy=6, z=FAKE, ldz=12, act=3, a=FAKE, lda=16, sa=FAKE, san=4, b=FAKE, ldb=16, sb=FAKE, sbn=12, da=FAKE, ldda=16,
              db=FAKE, lddb=16, dbias=NULL, M=4, F=6, K=16, mode=1, type=0, ws=FAKE, n=1 << 20):
    return niti.lib().niti_gated_bwd(dy, lddy, z, ldz, act, a, lda, sa, san, b, ldb, sb, sbn, da, ldda, db, lddb, dbias, M, F, K, mode, 0, 0,
                                     type, ws, n, None)


def test_gated_backward_rejects():
    assert gated_bwd(M=-1) == -2 and gated_bwd(F=-1) == -2 and gated_bwd(type=3) == -6 and gated_bwd(act=4) == -6 and gated_bwd(mode=0) == -6
    assert gated_bwd(M=1 << 17) == -3 and gated_bwd(F=1 << 16) == -3 and gated_bwd(K=1 << 22) == -3
    for name in ("dy", "z", "sa", "sb", "a", "b"):
        assert gated_bwd(**{name: NULL}) == -1, name
    assert gated_bwd(act=0, z=NULL) == -1                      # a gate without an activation multiplies all the same
    assert gated_bwd(san=2) == -2 and gated_bwd(sbn=6) == -2 and gated_bwd(lddy=5) == -2 and gated_bwd(ldz=11) == -2
    assert gated_bwd(ldda=0) == -2 and gated_bwd(lddb=15) == -2
    assert gated_bwd(ws=NULL) == -4 and gated_bwd(n=64) == -4 and gated_bwd(ws=ODD) == -6
    assert gated_bwd(da=NULL, db=NULL) == 0                     # nothing asked for


def emb_fwd(table=FAKE, ldt=8, tt=0, scale=NULL, tok=FAKE, out=FAKE, ldo=8, M=4, V=5, D=8, alpha=1.0, type=0):
    return niti.lib().niti_embedding_fwd(table, ldt, tt, scale, tok, out, ldo, M, V, D, alpha, type, None)


def test_embedding_forward_rejects():
    assert emb_fwd(M=-1) == -2 and emb_fwd(V=0) == -2 and emb_fwd(D=0) == -2
    assert emb_fwd(type=3) == -6 and emb_fwd(tt=4) == -6 and emb_fwd(alpha=INF) == -6 and emb_fwd(alpha=NAN) == -6
    assert emb_fwd(M=1 << 31) == -3 and emb_fwd(V=1 << 31) == -3 and emb_fwd(D=1 << 22) == -3
    for name in ("table", "tok", "out"):
        assert emb_fwd(**{name: NULL}) == -1, name
    assert emb_fwd(tt=3) == -1 and emb_fwd(scale=FAKE) == -1
    assert emb_fwd(ldt=7) == -2 and emb_fwd(ldo=7) == -2 and emb_fwd(ldo=0) == -2
    assert emb_fwd(M=0, table=NULL) == 0


def emb_bwd(dy=FAKE, lddy=8, type=0, tok=FAKE, dt=FAKE, ldt=8, gt=0, M=4, V=5, D=8, alpha=1.0, acc=0, ws=FAKE, n=1 << 20):
    return niti.lib().niti_embedding_bwd(dy, lddy, type, tok, dt, ldt, gt, M, V, D, alpha, acc, ws, n, None)


def test_embedding_backward_rejects():
    assert emb_bwd(M=-1) == -2 and emb_bwd(V=0) == -2 and emb_bwd(D=0) == -2
    assert emb_bwd(type=3) == -6 and emb_bwd(gt=3) == -6 and emb_bwd(alpha=NAN) == -6
    assert emb_bwd(M=(1 << 22) + 1) == -3 and emb_bwd(V=1 << 31) == -3 and emb_bwd(D=1 << 22) == -3
    for name in ("dy", "tok", "dt"):
        assert emb_bwd(**{name: NULL}) == -1, name
    assert emb_bwd(lddy=7) == -2 and emb_bwd(ldt=0) == -2
    assert emb_bwd(ws=NULL) == -4 and emb_bwd(n=64) == -4 and emb_bwd(ws=ODD) == -6
    assert emb_bwd(M=0, dy=NULL, dt=NULL, acc=1) == 0


def logprobs(x=FAKE, ldx=40, tok=FAKE, logp=FAKE, lse=NULL, ent=NULL, tv=FAKE, ti=FAKE, M=3, V=40, top=4, scale=1.0, type=0, ws=NULL, n=0):
    return niti.lib().niti_token_logprobs(x, ldx, tok, logp, lse, ent, tv, ti, M, V, top, scale, type, ws, n, None)


def test_logprobs_rejects():
    assert logprobs(M=-1) == -2 and logprobs(V=0) == -2 and logprobs(top=-1) == -2 and logprobs(top=41) == -2
    assert logprobs(type=3) == -6
    for s in (0.0, -1.0, INF, NAN):
        assert logprobs(scale=s) == -6
    assert logprobs(M=1 << 31) == -3 and logprobs(V=1 << 22) == -3 and logprobs(V=100, ldx=100, top=65) == -3
    assert logprobs(x=NULL) == -1 and logprobs(tok=NULL) == -1 and logprobs(logp=NULL) == -1 and logprobs(top=0) == -1
    assert logprobs(tv=NULL, ti=NULL) == -1 and logprobs(ldx=39) == -2
    wide = 1 << 20
    need = niti.workspace_bytes(niti.OP_TOKEN_LOGPROBS, None, 3, wide, 4)
    assert need > 0 and niti.workspace_bytes(niti.OP_TOKEN_LOGPROBS, None, 3, 4000, 4) == 0
    assert logprobs(V=wide, ldx=wide) == -4 and logprobs(V=wide, ldx=wide, ws=FAKE, n=16) == -4 and logprobs(V=wide, ldx=wide, ws=ODD, n=need) == -6
    assert logprobs(M=0, x=NULL) == 0


def distill_fwd(x=FAKE, ldx=40, tv=FAKE, ldt=4, tt=0, ti=FAKE, ldi=4, loss=FAKE, lse=NULL, dloss=NULL, dn=0, dx=NULL, lddx=0, M=3, V=40,
                top=4, scale=1.0, type=0, ws=NULL, n=0):
    return niti.lib().niti_distill_fwd(x, ldx, tv, ldt, tt, ti, ldi, loss, lse, dloss, dn, dx, lddx, M, V, top, scale, type, ws, n, None)


def distill_bwd(x=FAKE, ldx=40, tv=FAKE, ldt=4, tt=0, ti=FAKE, ldi=4, lse=FAKE, dloss=NULL, dn=0, dx=FAKE, lddx=40, M=3, V=40, top=4,
                scale=1.0, type=0):
    return niti.lib().niti_distill_bwd(x, ldx, tv, ldt, tt, ti, ldi, lse, dloss, dn, dx, lddx, M, V, top, scale, type, None)


def test_distill_rejects():
    for call in (distill_fwd, distill_bwd):
        assert call(M=-1) == -2 and call(V=0) == -2 and call(top=0) == -2 and call(type=3) == -6 and call(tt=-1) == -6
        for s in (0.0, -1.0, INF, NAN):
            assert call(scale=s) == -6
        assert call(M=1 << 31) == -3 and call(V=1 << 22) == -3 and call(top=257, ldt=257, ldi=257) == -3
        assert call(x=NULL) == -1 and call(tv=NULL) == -1 and call(ti=NULL) == -1
        assert call(ldx=39) == -2 and call(ldt=3) == -2 and call(ldi=3) == -2 and call(dx=FAKE, lddx=39) == -2
        assert call(dx=FAKE, lddx=40, dloss=FAKE, dn=2) == -2
        assert call(M=0, x=NULL) == 0
    assert distill_fwd(loss=NULL) == -1 and distill_fwd(dloss=FAKE, dn=1) == -1
    assert distill_bwd(lse=NULL) == -1 and distill_bwd(dx=NULL) == -1
    wide = 1 << 20
    need = niti.workspace_bytes(niti.OP_DISTILL_FWD, None, 3, wide)
    assert need > 0 and niti.workspace_bytes(niti.OP_DISTILL_FWD, None, 3, 4000) == 0
    assert distill_fwd(V=wide, ldx=wide) == -4 and distill_fwd(V=wide, ldx=wide, ws=ODD, n=need) == -6


def test_workspace_sizes():
    assert niti.workspace_bytes(niti.OP_GATED_FWD, None, 512, 512, 512) == 0
    assert niti.workspace_bytes(niti.OP_GATED_FWD, None, 4000, 4000, 4001) >= (4000 + 8000) * 4001
    assert niti.workspace_bytes(niti.OP_GATED_BWD, None, 33, 17, 50) >= 33 * 48 + 34 * 48 + 50 * (48 + 48)
    assert niti.workspace_bytes(niti.OP_GATED_BWD, None, 0, 17, 50) == 0 == niti.workspace_bytes(niti.OP_GATED_BWD, None, 4, 1 << 16, 50)
    assert niti.workspace_bytes(niti.OP_EMBEDDING_BWD, None, 100, 50, 8) > 0
    for m, v, d in ((0, 50, 8), (10, 0, 8), (10, 50, 0), ((1 << 22) + 1, 50, 8)):
        assert niti.workspace_bytes(niti.OP_EMBEDDING_BWD, None, m, v, d) == 0
    assert niti.workspace_bytes(niti.OP_TOKEN_LOGPROBS, None, 3, 1 << 20, 65) == 0 == niti.workspace_bytes(niti.OP_DISTILL_FWD, None, 3, 1 << 22)


def test_binding_takes_device_tensors_only():
    x, t = torch.zeros(2, 4), torch.zeros(2, dtype=torch.int32)
    q, s = x.to(torch.int8), torch.ones(2)
    for call in (lambda: niti.gated_fwd(q, q, x, s, s), lambda: niti.gated_bwd(x, x, q, q, s, s, None), lambda: niti.embedding_fwd(x, t, x),
                 lambda: niti.embedding_bwd(x, t, x, None), lambda: niti.token_logprobs(x, lse=s),
                 lambda: niti.distill_fwd(x, x, t.view(2, 1), s), lambda: niti.distill_bwd(x, x, t.view(2, 1), s, s, x)):
        with pytest.raises(TypeError):
            call()


@pytest.mark.parametrize("v", [30000, 40000, 65537, 100000, 131073, 262145, 1 << 20])
def test_workspace_of_many_rows_does_for_fewer(v):
    """A batch's workspace, sized once, serves the smaller last batch too."""
    rows = sorted(set(range(1, 200)) | {255, 256, 257, 511, 512, 513, 1000, 4096})
    for op, top in ((niti.OP_TOKEN_LOGPROBS, 0), (niti.OP_TOKEN_LOGPROBS, 20), (niti.OP_DISTILL_FWD, 0)):
        need = [niti.workspace_bytes(op, None, m, v, top) for m in rows]
        assert need == sorted(need)


@pytest.mark.parametrize("d", [64, 1000, 4096])
def test_workspace_of_many_tokens_does_for_fewer(d):
    need = [niti.workspace_bytes(niti.OP_EMBEDDING_BWD, None, m, 32000, d) for m in (1, 100, 4096, 8191, 8192, 8193, 16384, 32768, 32769, 100000)]
    assert need == sorted(need)
