"""The feed-forward block's and the optimiser's own work, without a GPU: a stand-in for the binding does the operators by their definitions (oracle/f8.py, oracle/ffn.py), reading
the memory that the calls name and nothing else."""
import copy
import io

import numpy as np
import pytest
import torch

from oracle import f8, ffn
from paper_1611_08035_b200 import adamw, binding, ffn8, layer8
from test_layer8 import BF, StandIn, columns, np64, off


class StandInFfn(StandIn):
    ACT_NONE, ACT_GRADIENT = binding.ACT_NONE, binding.ACT_GRADIENT

    def b2_rmsnorm_f8(self, d, t, *args):
        *args, rstd = args
        super().b2_rmsnorm_f8(d, t, *args, torch.empty(t) if rstd is None else rstd)

    def b2_act_backward_workspace_bytes(self, d, t):
        return 0

    def b2_gemm_f8_act(self, ta, tb, m, n, k, alpha, A, lda, SA, ldsa, ba, B, ldb, SB, ldsb, bb, act, bias, z, ldz, r, ldr, c, ldc, q, ldq, s, lds, ws):
        v = torch.empty(n, m, dtype=torch.float64)
        super().b2_gemm_f8(ta, tb, m, n, k, alpha, A, lda, SA, ldsa, ba, B, ldb, SB, ldsb, bb, 0.0, v, m, ws)
        self.calls[-1] = "act" + ta
        v, kind = v.numpy(), ffn.ACTS[act & 15]
        if act & 16:
            assert bias is None
            v = v * (ffn.act_slope(np64(columns(z, n, m, ldz)), kind) if act & 15 else 1.0)
        else:
            v = v + (0 if bias is None else np64(columns(bias, 1, m, m)[0]))
            if z is not None:
                columns(z, n, m, ldz).copy_(torch.from_numpy(v))
            v = ffn.act(v, kind)
        v = v + (0 if r is None else np64(columns(r, n, m, ldr)))
        if c is not None:
            columns(c, n, m, ldc).copy_(torch.from_numpy(v))
        self.quantised(v, q, ldq, s, lds)

    def quantised(self, v, q, ldq, s, lds):
        if q is not None:
            qv, sv = f8.quantise(v)
            columns(q, *qv.shape, ldq).copy_(torch.from_numpy(qv))
            columns(s, *sv.shape, lds).copy_(torch.from_numpy(sv))

    def b2_act_backward(self, d, t, act, dy, lddy, z, ldz, dz, lddz, q, ldq, s, lds, db, ws):
        self.called("act_backward")
        assert act == 0 and dz is None
        v = np64(columns(dy, t, d, lddy))
        self.quantised(v, q, ldq, s, lds)
        if db is not None:
            columns(db, 1, d, d).copy_(torch.from_numpy(v.sum(0)[None]))


@pytest.fixture
def ops(monkeypatch):
    s = StandInFfn()
    for module in (layer8, ffn8):
        monkeypatch.setattr(module, "b2", s)
    return s


def make(d=256, f=384, t=6, act="gelu"):
    torch.manual_seed(0)
    block = ffn8.FeedForward8(d, f, act, device="cpu")
    with torch.no_grad():
        block.up_bias += 0.3 * torch.randn(f)
    return block, *(torch.randn(t, d).to(BF).requires_grad_() for _ in range(2))


def test_stand_in_gives_the_block(ops):
    block, x, r = make()
    y = block(x, r)
    y.backward(torch.ones_like(y))
    p = {n: v.detach().float().requires_grad_() for n, v in block.named_parameters()}
    h = x.detach().float() + r.detach().float()
    n = h * torch.rsqrt(h.square().mean(1, keepdim=True) + block.eps) * p["norm_weight"]
    want = torch.nn.functional.gelu(n @ p["up"].t() + p["up_bias"]) @ p["down"].t() + p["down_bias"]
    want.backward(torch.ones_like(want))
    assert off(y.float() - h, want) < 0.12 and torch.equal(x.grad, r.grad)
    for name, v in block.named_parameters():
        assert off(v.grad, p[name].grad) < 0.13, name
    # the norm, two products; the gradient's quantisation, its product, the first bias's gradient, two weight gradients, the product before the norm and the norm
    assert ops.calls[2:] == ["norm", "actT", "actT", "act_backward", "wgrad", "actN", "act_backward", "wgrad", "gemmN", "norm_backward"]


def test_eight_bit_weights_follow(ops):
    block, x, _ = make()
    with torch.no_grad():
        first = block(x)
        assert ops.calls.count("quant") == 2
        block(x)
        assert ops.calls.count("quant") == 2
        block.down.mul_(-2.0)
        changed = block(x)
        assert ops.calls.count("quant") == 4 and not torch.equal(first, changed)
        block.up.data = block.up.data * 3.0  # no new version
        assert not torch.equal(block(x), changed) and ops.calls.count("quant") == 6
        assert torch.equal(copy.deepcopy(block)(x), block(x))
        block.double().float()
        block.norm_weight.data = block.norm_weight.data.to(BF)
        block(x)
        assert set(block.state_dict()) == {"norm_weight", "up", "down", "up_bias", "down_bias"}


def test_second_order_gradients_are_refused(ops):
    block, x, r = make()
    (g,) = torch.autograd.grad(block(x, r).float().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        g.float().square().sum().backward()


def test_captures(ops, monkeypatch):
    """What a capture made is no one else's, what it reads stays, and it is refused while an eager graph from another stream lives."""
    block, x, r = make()
    y = block(x, r)
    now = [True]
    monkeypatch.setattr(ffn8, "capturing", lambda x: now[0])
    block._graphs[0] = (block._graphs[0][0], 7)  # as if from another stream
    with pytest.raises(RuntimeError, match="alive"):
        block(x, r)
    with torch.no_grad():
        block(x, r)  # no gradients, nothing to add up
    del y
    eager = ops.calls.count("quant")
    old = block._quantised["up"][0]
    block(x, r)
    assert ops.calls.count("quant") == eager and any(q[0] is old for q in block._captured)
    block.requantise()
    assert any(q[0] is old for q in block._captured)
    block(x, r)
    assert ops.calls.count("quant") == eager + 2
    now[0] = False
    block(x, r)
    assert ops.calls.count("quant") == eager + 4
    y = block(x, r)
    assert ops.calls.count("quant") == eager + 4
    torch.save(block, io.BytesIO())
    assert torch.equal(copy.deepcopy(block)(x, r), y)


def test_refusals(ops):
    block, x, r = make()
    for bad in (x[:, :255], x.float(), x[0]):
        with pytest.raises(ValueError):
            block(bad)
    with pytest.raises(ValueError):
        block(x, r[:3])
    block.up_bias = torch.nn.Parameter(torch.zeros(7))
    with pytest.raises(ValueError):
        block(x)
    assert "norm" not in ops.calls


def test_optimiser_hands_over_what_belongs_together(monkeypatch):
    calls = []

    class Take:
        @staticmethod
        def b2_adamw(p, g, m, v, sm, sv, lr, b1, b2, eps, wd, step, seed, scale):
            calls.append((len(p), lr, b1, b2, eps, wd, step, seed, [x.dtype for x in m], [None if x is None else x.numel() for x in sm]))

    monkeypatch.setattr(adamw, "b2", Take)
    a, b, c = (torch.nn.Parameter(torch.zeros(n)) for n in (5000, 10, 300))
    opt = adamw.AdamW([{"params": [a, b]}, {"params": [c], "lr": 0.5}], lr=0.1)
    versions = [p._version for p in (a, b, c)]
    a.grad, c.grad = torch.ones(5000), torch.ones(300)
    opt.step()
    b.grad = torch.ones(10)
    opt.step()
    e4m3, f32 = torch.float8_e4m3fn, torch.float32
    assert calls == [(1, 0.1, 0.9, 0.999, 1e-8, 1e-2, 1, 0, [e4m3], [40]), (1, 0.5, 0.9, 0.999, 1e-8, 1e-2, 1, 1 << 32, [f32], [None]),
                     (1, 0.1, 0.9, 0.999, 1e-8, 1e-2, 2, 0, [e4m3], [40]), (1, 0.1, 0.9, 0.999, 1e-8, 1e-2, 1, 0, [f32], [None]), (1, 0.5, 0.9, 0.999, 1e-8, 1e-2, 2, 1 << 32, [f32], [None])]
    assert [p._version - v for p, v in zip((a, b, c), versions)] == [2, 1, 2]
    a.grad = torch.ones(5000).to_sparse()
    with pytest.raises(RuntimeError):
        opt.step()
    with pytest.raises(ValueError):
        adamw.AdamW([torch.nn.Parameter(torch.zeros(4, 6).t())])
    done = len(calls)
    monkeypatch.setattr(adamw, "capturing", lambda x: True)
    for capturable in (False, True):  # its number would be the replay's, its first states too
        opt = adamw.AdamW([c], capturable=capturable)
        with pytest.raises(RuntimeError, match="capture"):
            opt.step()
    assert len(calls) == done
    with pytest.raises(ValueError):
        adamw.AdamW([a], betas=(0.9, 1.0))
    assert np.isfinite(float(a.detach().sum()))
