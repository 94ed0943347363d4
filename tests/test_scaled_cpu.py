"""Operators on int8 rows: argument checks on the host, before anything is launched."""
import ctypes

import pytest
import torch

from paper_2009_13108_amd import niti

FAKE = ctypes.c_void_p(0x100000)   # never dereferenced: every call below fails validation
NULL = None


def test_struct_layout_matches_header():
    assert ctypes.sizeof(niti.AdamWTensor) == 9 * 8
    assert niti.AdamWTensor.n.offset == 64


def test_workspace_sizes():
    assert niti.workspace_bytes(niti.OP_RMSNORM_BWD, None, 100, 64) > 0
    assert niti.workspace_bytes(niti.OP_RMSNORM_BWD, None, 0, 64) == 0
    assert niti.workspace_bytes(niti.OP_LINEAR_BWD, None, 33, 17, 50) >= 33 * 32 + 17 * 48 + 50 * (32 + 48)
    assert niti.workspace_bytes(niti.OP_LINEAR_BWD, None, 0, 17, 50) == 0
    assert niti.workspace_bytes(niti.OP_LINEAR_FWD, None, 8192, 8192, 8192) == 0


def norm_fwd(x=FAKE, ldx=8, res=NULL, ldres=0, gain=FAKE, gt=0, h=NULL, ldh=0, y=FAKE, ldy=8, q=NULL, ldq=0, scale=NULL, rstd=NULL,
             M=4, D=8, eps=1e-6, type=0):
    return niti.lib().niti_rmsnorm_fwd(x, ldx, res, ldres, gain, gt, h, ldh, y, ldy, q, ldq, scale, rstd, M, D, eps, type, None)


def test_norm_forward_rejects():
    assert norm_fwd(M=-1) == -2 and norm_fwd(D=0) == -2
    assert norm_fwd(type=3) == -6 and norm_fwd(gt=-1) == -6 and norm_fwd(eps=-1.0) == -6 and norm_fwd(eps=float("nan")) == -6
    assert norm_fwd(x=NULL) == -1 and norm_fwd(gain=NULL) == -1
    assert norm_fwd(q=FAKE, ldq=8) == -1 and norm_fwd(scale=FAKE) == -1
    assert norm_fwd(ldx=7) == -2 and norm_fwd(ldy=7) == -2 and norm_fwd(ldy=0) == -2 and norm_fwd(res=FAKE, ldres=-8) == -2
    assert norm_fwd(h=FAKE, ldh=4) == -2 and norm_fwd(ldx=1 << 22) == -2
    assert norm_fwd(M=1 << 31) == -3 and norm_fwd(D=1 << 22) == -3
    assert norm_fwd(M=0, x=NULL) == 0


def norm_bwd(dy=FAKE, lddy=8, h=FAKE, ldh=8, gain=FAKE, gt=0, rstd=FAKE, dh=NULL, lddh=0, dx=FAKE, lddx=8, dgain=NULL, M=4, D=8,
             type=0, ws=NULL, n=0):
    return niti.lib().niti_rmsnorm_bwd(dy, lddy, h, ldh, gain, gt, rstd, dh, lddh, dx, lddx, dgain, M, D, type, ws, n, None)


def test_norm_backward_rejects():
    assert norm_bwd(M=-1) == -2 and norm_bwd(D=0) == -2 and norm_bwd(type=9) == -6
    for name in ("dy", "h", "gain", "rstd", "dx"):
        assert norm_bwd(**{name: NULL}) == -1, name
    assert norm_bwd(lddx=4) == -2 and norm_bwd(dh=FAKE, lddh=7) == -2
    assert norm_bwd(dgain=FAKE) == -4 and norm_bwd(dgain=FAKE, ws=FAKE, n=16) == -4
    need = niti.workspace_bytes(niti.OP_RMSNORM_BWD, None, 4, 8)
    assert norm_bwd(dgain=FAKE, ws=ctypes.c_void_p(0x100002), n=need) == -6
    assert norm_bwd(M=0) == 0


def quant(x=FAKE, ldx=8, q=FAKE, ldq=8, scale=FAKE, y=NULL, ldy=0, M=4, D=8, mode=1, type=0):
    return niti.lib().niti_quantize_rows(x, ldx, q, ldq, scale, y, ldy, M, D, mode, 0, 0, type, None)


def test_quantize_rejects():
    assert quant(M=-1) == -2 and quant(D=0) == -2 and quant(mode=0) == -6 and quant(mode=3) == -6 and quant(type=5) == -6
    assert quant(x=NULL) == -1 and quant(q=NULL) == -1 and quant(scale=NULL) == -1
    assert quant(ldq=7) == -2 and quant(y=FAKE, ldy=2) == -2 and quant(M=0) == 0


def lin_fwd(a=FAKE, lda=16, sa=FAKE, san=4, b=FAKE, ldb=16, sb=FAKE, sbn=6, bias=NULL, bt=0, act=0, res=NULL, ldres=0, z=NULL, ldz=0,
            out=FAKE, ldout=6, M=4, N=6, K=16, type=0, ws=NULL, n=0):
    return niti.lib().niti_linear_fwd(a, lda, sa, san, b, ldb, sb, sbn, bias, bt, act, res, ldres, z, ldz, out, ldout, M, N, K, type, ws,
                                      n, None)


def test_linear_forward_rejects():
    assert lin_fwd(M=-1) == -2 and lin_fwd(N=-1) == -2 and lin_fwd(K=-1) == -2
    assert lin_fwd(type=3) == -6 and lin_fwd(act=4) == -6 and lin_fwd(act=-1) == -6 and lin_fwd(bias=FAKE, bt=7) == -6
    assert lin_fwd(K=1 << 17, lda=1 << 17, ldb=1 << 17) == -3 and lin_fwd(N=1 << 22) == -3 and lin_fwd(M=1 << 31) == -3
    assert lin_fwd(a=NULL) == -1 and lin_fwd(b=NULL) == -1 and lin_fwd(out=NULL) == -1 and lin_fwd(sa=NULL) == -1 and lin_fwd(sb=NULL) == -1
    assert lin_fwd(san=3) == -2 and lin_fwd(sbn=2) == -2
    assert lin_fwd(lda=15) == -2 and lin_fwd(ldb=8) == -2 and lin_fwd(ldout=5) == -2 and lin_fwd(z=FAKE, ldz=0) == -2
    assert lin_fwd(res=FAKE, ldres=3) == -2 and lin_fwd(n=64) == -4
    assert lin_fwd(M=0, a=NULL) == 0 and lin_fwd(N=0, out=NULL) == 0


def lin_bwd(dy=FAKE, lddy=6, z=NULL, ldz=0, act=0, a=FAKE, lda=16, sa=FAKE, san=4, b=FAKE, ldb=16, sb=FAKE, sbn=6, da=FAKE, ldda=16,
            db=FAKE, lddb=16, dbias=NULL, M=4, N=6, K=16, mode=1, type=0, ws=FAKE, n=1 << 20):
    return niti.lib().niti_linear_bwd(dy, lddy, z, ldz, act, a, lda, sa, san, b, ldb, sb, sbn, da, ldda, db, lddb, dbias, M, N, K, mode, 0,
                                      0, type, ws, n, None)


def test_linear_backward_rejects():
    assert lin_bwd(M=-1) == -2 and lin_bwd(type=3) == -6 and lin_bwd(act=4) == -6 and lin_bwd(mode=0) == -6
    assert lin_bwd(M=1 << 17) == -3 and lin_bwd(N=1 << 17) == -3 and lin_bwd(K=1 << 22) == -3
    for name in ("dy", "sa", "sb", "a", "b"):
        assert lin_bwd(**{name: NULL}) == -1, name
    assert lin_bwd(act=3) == -1                               # no z
    assert lin_bwd(san=2) == -2 and lin_bwd(sbn=5) == -2 and lin_bwd(lddy=5) == -2 and lin_bwd(ldda=0) == -2 and lin_bwd(lddb=15) == -2
    assert lin_bwd(ws=NULL) == -4 and lin_bwd(n=64) == -4 and lin_bwd(ws=ctypes.c_void_p(0x100008)) == -6
    assert lin_bwd(da=NULL, db=NULL) == 0                     # nothing asked for


def step(tensors, count, p=0, g=0, bits=32, t=1, lr=1e-3, b1=0.9, b2=0.99, eps=1e-8, mode=1):
    return niti.lib().niti_adamw_step(tensors, count, p, g, bits, t, lr, b1, b2, eps, 0.0, None, mode, 0, None)


def test_adamw_rejects():
    row = (niti.AdamWTensor * 1)()
    row[0].n = 4
    assert step(row, -1) == -2 and step(NULL, 1) == -1 and step(row, 1) == -1
    row[0].m = row[0].v = row[0].g = 0x1000
    assert step(row, 1) == -1                                  # no parameter
    row[0].p = 0x1000
    assert step(row, 1, bits=8) == -1                          # no scales
    assert step(row, 1, bits=16) == -6 and step(row, 1, p=3) == -6 and step(row, 1, g=-1) == -6 and step(row, 1, t=0) == -6
    assert step(row, 1, b1=1.0) == -6 and step(row, 1, b2=-0.1) == -6 and step(row, 1, eps=-1.0) == -6 and step(row, 1, mode=0) == -6
    assert step(row, 1, lr=float("nan")) == -6
    row[0].n = -1
    assert step(row, 1) == -2
    row[0].n = 0
    assert step(row, 1) == 0 and step(NULL, 0) == 0            # nothing to do
    assert niti.lib().niti_adamw_read(row, 1, 7, None) == -6 and niti.lib().niti_adamw_read(NULL, 2, 0, None) == -1


def test_binding_takes_device_tensors_only():
    x, g = torch.zeros(2, 4), torch.ones(4)
    with pytest.raises(TypeError):
        niti.rmsnorm_fwd(x, g, y=x)
    with pytest.raises(TypeError):
        niti.quantize_rows(x, x.to(torch.int8), g)
    with pytest.raises(TypeError):
        niti.linear_fwd(x.to(torch.int8), x.to(torch.int8), x, g, g)
    with pytest.raises(TypeError):
        niti.adamw_plan([x], [x], [x], [x])
