"""Refusals of the 8-bit entry points: every illegal argument has its number, nothing is launched, no GPU is needed."""
import ctypes

import pytest
import torch

F = ctypes.c_void_p(4096)  # never dereferenced: every call fails its argument check first
f = ctypes.c_float


def test_rmsnorm_refusals(b2):
    good = dict(d=200, t=3, type=2, X=F, ldx=200, R=F, ldr=200, w=F, eps=1e-5, H=F, ldh=200, Q=F, ldq=200, S=F, lds=2)

    def call(**kw):
        a = {**good, **kw}
        return b2.lib().b2_rmsnorm_f8(*[f(v) if k == "eps" else v for k, v in a.items()], None, None)

    for number, bad in [(1, dict(d=-1)), (2, dict(t=-1)), (3, dict(type=0)), (4, dict(X=None)), (5, dict(ldx=199)), (7, dict(ldr=199)),
                        (8, dict(w=None)), (9, dict(eps=-1.0)), (9, dict(eps=float("nan"))), (11, dict(ldh=199)), (12, dict(Q=None)),
                        (13, dict(ldq=199)), (14, dict(S=None)), (15, dict(lds=1))]:
        assert call(**bad) == -number, bad
    assert call(t=0, X=None, w=None, Q=None, S=None) == 0 and call(d=0, X=None, w=None, Q=None, S=None, lds=1) == 0


def test_rmsnorm_backward_refusals(b2):
    good = dict(d=200, t=3, type=1, DY=F, lddy=200, H=F, ldh=200, rstd=F, w=F, DH=F, lddh=200, DX=F, lddx=200, dw=F, ws=F, n=1 << 30)

    def call(**kw):
        return b2.lib().b2_rmsnorm_backward(*{**good, **kw}.values(), None)

    for number, bad in [(1, dict(d=-1)), (2, dict(t=-1)), (3, dict(type=3)), (4, dict(DY=None)), (5, dict(lddy=199)), (6, dict(H=None)),
                        (7, dict(ldh=199)), (8, dict(rstd=None)), (9, dict(w=None)), (11, dict(lddh=199)), (12, dict(DX=None)),
                        (13, dict(lddx=199)), (14, dict(dw=None))]:
        assert call(**bad) == -number, bad
    assert call(ws=None) == 1003 and call(n=16) == 1003 and call(ws=ctypes.c_void_p(4100)) == 1003
    assert call(d=0, DY=None, H=None, rstd=None, w=None, DX=None, dw=None) == 0
    assert b2.b2_rmsnorm_backward_workspace_bytes(200, 0) == 0 and b2.b2_rmsnorm_backward_workspace_bytes(200, 3) % 256 == 0


def test_quant_refusals(b2):
    good = dict(d=200, t=3, block=1, type=2, X=F, ldx=200, Q=F, ldq=200, S=F, lds=2)

    def call(**kw):
        return b2.lib().b2_quant_f8(*{**good, **kw}.values(), None)

    for number, bad in [(1, dict(d=-1)), (2, dict(t=-1)), (3, dict(block=64)), (4, dict(type=7)), (5, dict(X=None)), (6, dict(ldx=199)),
                        (7, dict(Q=None)), (8, dict(ldq=199)), (9, dict(S=None)), (10, dict(lds=1))]:
        assert call(**bad) == -number, bad
    assert call(t=0, X=None, Q=None, S=None) == 0


def test_gemm_refusals(b2):
    good = dict(ta=b"T", tb=b"N", m=300, n=5, k=200, alpha=1.0, A=F, lda=208, SA=F, ldsa=2, ba=128, ta_=0, B=F, ldb=208, SB=F, ldsb=2, bb=1,
                tb_=0, beta=0.0, C=F, ldc=300, tc=2, ws=None, n_ws=0)

    def call(**kw):
        a = {**good, **kw}
        return b2.lib().b2_gemm_f8(*[f(v) if k in ("alpha", "beta") else v for k, v in a.items()], None)

    for number, bad in [(1, dict(ta=b"X")), (2, dict(tb=b"Q")), (3, dict(m=-1)), (4, dict(n=-1)), (5, dict(k=-1)), (7, dict(A=None)),
                        (8, dict(lda=199)), (8, dict(ta=b"N", lda=299)), (9, dict(SA=None)), (10, dict(ldsa=1)), (10, dict(ta=b"N", lda=304, ldsa=2)),
                        (11, dict(ba=64)), (12, dict(ta_=2)), (13, dict(B=None)), (14, dict(ldb=199)), (15, dict(SB=None)), (16, dict(ldsb=1)),
                        (16, dict(tb=b"T", ldsb=4)), (17, dict(bb=0)), (18, dict(tb_=-1)), (20, dict(C=None)), (21, dict(ldc=299)), (22, dict(tc=0))]:
        assert call(**bad) == -number, bad
    assert call(n=0, B=None, SB=None, C=None) == 0
    # an operand that is not aligned needs a workspace, and says how much
    assert call(lda=201) == 1003 and call(A=ctypes.c_void_p(4097)) == 1003
    assert b2.lib().b2_gemm_f8_workspace_bytes(b"T", b"N", 300, 5, 200, F, 201, F, 208) == -(-208 * 300 // 256) * 256
    assert b2.lib().b2_gemm_f8_workspace_bytes(b"T", b"N", 300, 5, 200, F, 208, F, 208) == 0
    assert call(m=2**31, lda=2**31, ldc=2**31) == 1004


def test_wgrad_refusals(b2):
    good = dict(m=300, n=40, k=5, alpha=1.0, Q=F, ldq=304, S=F, lds=3, Y=F, ldy=40, beta=0.0, C=F, ldc=300, tc=1, ws=None, n_ws=0)

    def call(**kw):
        a = {**good, **kw}
        return b2.lib().b2_wgrad_f8(*[f(v) if k in ("alpha", "beta") else v for k, v in a.items()], None)

    for number, bad in [(1, dict(m=-1)), (2, dict(n=-1)), (3, dict(k=-1)), (5, dict(Q=None)), (6, dict(ldq=299)), (7, dict(S=None)),
                        (8, dict(lds=2)), (9, dict(Y=None)), (10, dict(ldy=39)), (12, dict(C=None)), (13, dict(ldc=299)), (14, dict(tc=9))]:
        assert call(**bad) == -number, bad
    assert call(m=0, Q=None, S=None, C=None) == 0
    assert call(ldq=301) == 1003 and call(ldy=41) == 1003
    assert b2.lib().b2_wgrad_f8_workspace_bytes(300, 40, 5, F, 304, F, 40) == 0


def test_binding_refuses_wrong_types(b2):
    x = torch.zeros(4, 128)
    q, s = torch.zeros(4, 128, dtype=torch.float8_e4m3fn), torch.zeros(4, 1, dtype=torch.uint8).view(torch.float8_e8m0fnu)
    with pytest.raises(TypeError):
        b2.b2_quant_f8(128, 4, 1, x.half(), 128, q, 128, s, 1)
    with pytest.raises(TypeError):  # host tensors
        b2.b2_quant_f8(128, 4, 1, x, 128, q, 128, s, 1)
    with pytest.raises(TypeError):
        b2.b2_gemm_f8("T", "N", 4, 4, 128, 1.0, q, 128, s.view(torch.uint8), 1, 1, q, 128, s, 1, 1, 0.0, x, 4)
    with pytest.raises(TypeError):
        b2.b2_wgrad_f8(128, 4, 4, 1.0, q, 128, s, 1, x, 4, 0.0, x, 128)
