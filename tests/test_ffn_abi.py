"""Refusals of the feed-forward block's entry points: every illegal argument has its number, nothing is launched, no GPU is needed."""
import ctypes

import pytest
import torch

F = ctypes.c_void_p(4096)  # never dereferenced: every call fails its argument check first, or has nothing to do
f = ctypes.c_float


def test_gemm_act_refusals(b2):
    good = dict(ta=b"T", tb=b"N", m=300, n=5, k=200, alpha=1.0, A=F, lda=208, SA=F, ldsa=2, ba=128, ta_=0, B=F, ldb=208, SB=F, ldsb=2, bb=1, tb_=0,
                act=2, bias=F, Z=F, ldz=300, R=F, ldr=300, C=F, ldc=300, type=2, Q=F, ldq=300, S=F, lds=3, ws=None, n_ws=0)

    def call(**kw):
        a = {**good, **kw}
        return b2.lib().b2_gemm_f8_act(*[f(v) if k == "alpha" else v for k, v in a.items()], None)

    for number, bad in [(1, dict(ta=b"X")), (2, dict(tb=b"Q")), (3, dict(m=-1)), (4, dict(n=-1)), (5, dict(k=-1)), (7, dict(A=None)), (8, dict(lda=199)),
                        (9, dict(SA=None)), (10, dict(ldsa=1)), (11, dict(ba=64)), (12, dict(ta_=2)), (13, dict(B=None)), (14, dict(ldb=199)),
                        (15, dict(SB=None)), (16, dict(ldsb=1)), (17, dict(bb=0)), (18, dict(tb_=-1)), (19, dict(act=5)), (19, dict(act=-1)), (19, dict(act=32)),
                        (20, dict(act=2 | 16)), (21, dict(act=2 | 16, bias=None, Z=None)), (22, dict(ldz=299)), (24, dict(ldr=299)), (25, dict(C=None, Q=None)),
                        (26, dict(ldc=299)), (27, dict(type=0)), (29, dict(ldq=299)), (30, dict(S=None)), (31, dict(lds=2))]:
        assert call(**bad) == -number, bad
    assert call(n=0, B=None, SB=None, C=None, Q=None) == 0 and call(m=0, A=None, ldz=1, ldr=1, ldc=1, ldq=1, lds=1, C=None, Q=None) == 0
    assert call(lda=201) == 1003 and call(m=2**31, Z=None, R=None, Q=None, lda=2**31, ldc=2**31) == 1004


def test_act_backward_refusals(b2):
    good = dict(d=200, t=3000, type=1, act=4, DY=F, lddy=200, Z=F, ldz=200, DZ=F, lddz=200, Q=F, ldq=200, S=F, lds=2, db=F, ws=F, n=1 << 30)

    def call(**kw):
        return b2.lib().b2_act_backward(*{**good, **kw}.values(), None)

    for number, bad in [(1, dict(d=-1)), (2, dict(t=-1)), (3, dict(type=3)), (4, dict(act=16)), (4, dict(act=5)), (5, dict(DY=None)), (6, dict(lddy=199)), (7, dict(Z=None)),
                        (8, dict(ldz=199)), (10, dict(lddz=199)), (12, dict(ldq=199)), (13, dict(S=None)), (14, dict(lds=1))]:
        assert call(**bad) == -number, bad
    assert call(ws=None) == 1003 and call(n=16) == 1003 and call(ws=ctypes.c_void_p(4100)) == 1003
    assert call(d=0, DY=None, Z=None) == 0 and call(DZ=None, Q=None, db=None) == 0
    assert b2.b2_act_backward_workspace_bytes(200, 0) == 0 and b2.b2_act_backward_workspace_bytes(200, 8) == 0
    assert b2.b2_act_backward_workspace_bytes(200, 3000) % 256 == 0


def test_adamw_refusals(b2):
    good = dict(param=4096, grad=1 << 20, m=2 << 20, v=3 << 20, sm=4 << 20, sv=5 << 20, n=10, type_param=1, type_grad=2, state_bits=8, reserved=0)

    def call(tensors=None, count=None, lr=1e-3, b1=0.9, b2_=0.99, eps=1e-8, wd=0.1, step=1, seed=0, scale=None, lr_device=None, step_device=None, **kw):
        list_ = [{**good, **kw}] if tensors is None else tensors
        table = (b2._AdamwTensor * max(1, len(list_)))(*[b2._AdamwTensor(*t.values()) for t in list_])
        return b2.lib().b2_adamw(table, len(list_) if count is None else count, lr, b1, b2_, eps, wd, step, seed, scale, lr_device, step_device, None)

    inf, nan = float("inf"), float("nan")
    for number, bad in [(1, dict(param=None)), (1, dict(grad=None)), (1, dict(m=None)), (1, dict(v=None)), (1, dict(sm=None)), (1, dict(sv=None)), (1, dict(n=-1)),
                        (1, dict(type_param=0)), (1, dict(type_grad=3)), (1, dict(state_bits=16)), (1, dict(reserved=1)), (1, dict(param=4098)), (1, dict(grad=4097)),
                        (1, dict(state_bits=32, m=4097)), (2, dict(count=-1)), (3, dict(lr=nan)), (3, dict(lr=inf)), (4, dict(b1=1.0)), (4, dict(b1=-0.1)), (4, dict(b1=nan)),
                        (5, dict(b2_=1.0)), (5, dict(b2_=nan)), (6, dict(eps=-1.0)), (6, dict(eps=nan)), (7, dict(wd=inf)), (8, dict(step=0)), (8, dict(step=-3))]:
        assert call(**bad) == -number, bad
    assert b2.lib().b2_adamw(None, 1, 1e-3, 0.9, 0.99, 1e-8, 0.1, 1, 0, None, None, None, None) == -1
    assert call(tensors=[good, good]) == -1 and call(tensors=[good, {**good, "param": 4096 + 36}]) == -1  # the same memory twice
    assert call(tensors=[]) == 0 and call(n=0, param=None, grad=None) == 0 and b2.lib().b2_adamw(None, 0, 1e-3, 0.9, 0.99, 1e-8, 0.1, 1, 0, None, None, None, None) == 0
    many = [{**good, "param": 4096 + 64 * i} for i in range(50)]
    assert call(tensors=many + [many[7]]) == -1


def test_bindings_refuse_wrong_tensors(b2):
    x, h = torch.zeros(4, 128), torch.zeros(4, 128, dtype=torch.float16)
    q, s = torch.zeros(4, 128, dtype=torch.float8_e4m3fn), torch.zeros(4, 1, dtype=torch.uint8).view(torch.float8_e8m0fnu)
    with pytest.raises(TypeError):  # host tensors
        b2.b2_gemm_f8_act("T", "N", 4, 4, 128, 1.0, q, 128, s, 1, 1, q, 128, s, 1, 1, 0, None, None, 4, None, 4, x, 4, None, 0, None, 0)
    with pytest.raises(TypeError):
        b2.b2_gemm_f8_act("T", "N", 4, 4, 128, 1.0, q, 128, s, 1, 1, q, 128, s, 1, 1, 0, None, None, 4, None, 4, h, 4, None, 0, None, 0)
    with pytest.raises(TypeError):
        b2.b2_act_backward(128, 4, 0, x, 128, None, 0, None, 0, q, 128, s, 1, None)
    with pytest.raises(TypeError):
        b2.b2_adamw([x], [x], [x], [x], None, None, 1e-3, 0.9, 0.99, 1e-8, 0.0, 1)
    with pytest.raises(ValueError):
        b2.b2_adamw([x, x], [x], [x], [x], None, None, 1e-3, 0.9, 0.99, 1e-8, 0.0, 1)
