"""The 8-bit layer's own work, without a GPU: a stand-in for the binding does the operators by their definitions (oracle/f8.py), reading the
memory that the calls name and nothing else."""
import copy

import numpy as np
import pytest
import torch

from oracle import f8
from paper_1611_08035_b200 import layer8

BF, F32 = torch.bfloat16, torch.float32


def columns(x, t, d, ld):
    """t columns of d elements, ld apart, from where x begins; raises where they leave x's memory."""
    return torch.as_strided(x.view(torch.uint8) if x.element_size() == 1 else x, (t, d), (ld, 1))


def np64(x):
    return x.detach().to(torch.float64).numpy()


class StandIn:
    def __init__(self):
        self.calls, self.devices = [], []

    def called(self, name):
        self.calls.append(name)
        self.devices.append(layer8_device[-1] if layer8_device else None)

    def b2_quant_f8(self, d, t, block, x, ldx, q, ldq, s, lds):
        self.called("quant")
        qv, sv = f8.quantise(np64(columns(x, t, d, ldx)), block)
        columns(q, t, d, ldq).copy_(torch.from_numpy(qv))
        columns(s, *sv.shape, lds).copy_(torch.from_numpy(sv))

    def b2_rmsnorm_f8(self, d, t, x, ldx, r, ldr, w, eps, h, ldh, q, ldq, s, lds, rstd):
        self.called("norm")
        hv, rv, yv = f8.rmsnorm(np64(columns(x, t, d, ldx)), None if r is None else np64(columns(r, t, d, ldr)), np64(columns(w, 1, d, d)[0]), eps)
        if h is not None:
            columns(h, t, d, ldh).copy_(torch.from_numpy(hv))
        qv, sv = f8.quantise(yv)
        columns(q, t, d, ldq).copy_(torch.from_numpy(qv))
        columns(s, *sv.shape, lds).copy_(torch.from_numpy(sv))
        rstd.copy_(torch.from_numpy(rv))

    def b2_rmsnorm_backward_workspace_bytes(self, d, t):
        return 0

    def b2_gemm_f8_workspace_bytes(self, *a):
        return 0

    def b2_wgrad_f8_workspace_bytes(self, *a):
        return 0

    def b2_rmsnorm_backward(self, d, t, dy, lddy, h, ldh, rstd, w, dh, lddh, dx, lddx, dw, ws):
        self.called("norm_backward")
        a, b = f8.rmsnorm_backward(np64(columns(dy, t, d, lddy)), np64(columns(h, t, d, ldh)), np64(rstd), np64(columns(w, 1, d, d)[0]),
                                   None if dh is None else np64(columns(dh, t, d, lddh)))
        columns(dx, t, d, lddx).copy_(torch.from_numpy(a))
        dw.copy_(torch.from_numpy(b))

    def b2_gemm_f8(self, ta, tb, m, n, k, alpha, A, lda, SA, ldsa, ba, B, ldb, SB, ldsb, bb, beta, C, ldc, ws):
        self.called("gemm" + ta)
        assert tb == "N" and alpha == 1.0 and beta == 0.0
        rows, cols = (m, k) if ta == "T" else (k, m)
        qa, sa = f8.E4M3[columns(A, rows, cols, lda).numpy()], f8.e8m0(columns(SA, -(-rows // ba) if ta == "T" else -(-rows // 128), -(-cols // 128), ldsa).numpy())
        if ta == "N":
            qa, sa = qa.T, sa.T
        qb, sb = f8.E4M3[columns(B, n, k, ldb).numpy()], f8.e8m0(columns(SB, -(-n // bb), -(-k // 128), ldsb).numpy())
        columns(C, n, m, ldc).copy_(torch.from_numpy(f8.gemm(qa, sa, ba, qb, sb, bb)[0]))

    def b2_wgrad_f8(self, m, n, k, alpha, Q, ldq, S, lds, Y, ldy, beta, C, ldc, ws):
        self.called("wgrad")
        q, s = f8.E4M3[columns(Q, k, m, ldq).numpy()], f8.e8m0(columns(S, k, -(-m // 128), lds).numpy())
        columns(C, n, m, ldc).copy_(torch.from_numpy(f8.wgrad(q, s, np64(columns(Y, k, n, ldy)))[0]))


layer8_device = []


@pytest.fixture
def ops(monkeypatch):
    s = StandIn()
    monkeypatch.setattr(layer8, "b2", s)
    layer8_device.clear()
    return s


def make(d=256, n=128, t=5, seed=0):
    g = torch.Generator().manual_seed(seed)
    torch.manual_seed(seed)
    layer = layer8.NormLinear8(d, n, device="cpu")
    x, r = (torch.randn(t, d, generator=g).to(BF).requires_grad_() for _ in range(2))
    return layer, x, r


def reference(layer, x, r):
    h = x.float() + (0 if r is None else r.float())
    return h * torch.rsqrt(h.square().mean(1, keepdim=True) + layer.eps) * layer.norm_weight.float() @ layer.weight.float().t()


def off(a, b):
    return float((a.detach().float() - b.detach().float()).norm() / b.detach().float().norm())


def test_stand_in_gives_the_layer(ops):
    layer, x, r = make()
    y, h = layer(x, r)
    y.float().square().sum().backward()
    xf, rf = x.detach().float().requires_grad_(), r.detach().float().requires_grad_()
    want = reference(layer, xf, rf)
    want.square().sum().backward()
    assert off(y, want) < 2 * 0.037 and off(x.grad, xf.grad) < 0.1 and torch.equal(x.grad, r.grad)


def test_second_order_gradients_are_refused(ops):
    """The backward pass is made of operators without a gradient: a loss with a gradient in it must not quietly lose that part."""
    layer, x, r = make()
    y, _ = layer(x, r)
    (g,) = torch.autograd.grad(y.float().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        (y.float().sum() + g.float().square().sum()).backward()


def change_in_place(layer):
    with torch.no_grad():
        layer.weight.mul_(-2.0)
    return layer


def change_by_loading(layer):
    layer.load_state_dict({"norm_weight": layer.norm_weight.detach().clone(), "weight": layer.weight.detach() * -2.0})
    return layer


def change_by_another_parameter(layer):
    layer.weight = torch.nn.Parameter(layer.weight.detach() * -2.0)
    return layer


def change_of_a_copy(layer):
    return change_in_place(copy.deepcopy(layer))


def change_by_conversion(layer):  # what .to(), .cuda() and their kind do, here with a function that also changes the numbers
    return layer._apply(lambda p: p * -2.0 if p.dim() == 2 else p)


@pytest.mark.parametrize("change", [change_in_place, change_by_loading, change_by_another_parameter, change_of_a_copy, change_by_conversion])
def test_weight_in_8_bits_follows_the_weight(ops, change):
    """Whatever changes the weight without a word to the layer: the products read the new one."""
    layer, x, r = make()
    layer(x, r)
    layer = change(layer)
    y, _ = layer(x, r)
    assert off(y, reference(layer, x, r)) < 2 * 0.037


def test_weight_in_8_bits_is_made_once(ops):
    layer, x, r = make()
    before = layer.weight.detach().clone()
    for _ in range(3):
        y, _ = layer(x, r)
        y.float().sum().backward()
    assert ops.calls.count("norm") == 3 and ops.calls.count("quant") == 1 + 3  # the weight's, and each step's gradient
    layer.requantise()
    assert ops.calls.count("quant") == 5 and torch.equal(layer.weight, before)


def test_state_is_the_weights_alone(ops):
    layer, x, r = make()
    assert set(layer.state_dict()) == {"norm_weight", "weight"} and len(list(layer.parameters())) == 2


@pytest.mark.parametrize("transposed", [False, True])
def test_quantise_reads_any_layout(ops, transposed):
    """What the operator is given are columns one after the other, whatever the tensor's strides: nothing beyond its memory, the same numbers."""
    x = torch.randn(130, 200, generator=torch.Generator().manual_seed(1))
    view = x.t().contiguous().t() if transposed else x[:1].expand(130, 200)
    q, s = layer8.quantise(view, 128)
    want_q, want_s = f8.quantise(np64(view), 128)
    assert np.array_equal(q.view(torch.uint8).numpy(), want_q) and np.array_equal(s.view(torch.uint8).numpy(), want_s)


def test_shapes_that_do_not_fit_are_refused(ops):
    """Every operand's extent comes from x and the weight: another tensor's would be read beyond its end."""
    layer, x, r = make(256, 128, 5)
    for bad_x, bad_r in [(x, r[:1]), (x, r[:, :128]), (x, r[:4]), (x[:, :255], None), (torch.zeros(5, 257, dtype=BF), None), (x[0], None), (x[None], None),
                         (x, r[None]), (x.detach().to("meta"), None)]:
        with pytest.raises(ValueError):
            layer(bad_x, bad_r)
    layer.norm_weight = torch.nn.Parameter(torch.ones(1, dtype=BF))
    with pytest.raises(ValueError):
        layer(x, r)
    assert "norm" not in ops.calls


def test_strided_norm_weight(ops):
    layer, x, r = make(256, 128, 5)
    wide = torch.randn(512, generator=torch.Generator().manual_seed(2)).to(BF)
    layer.norm_weight = torch.nn.Parameter(wide[::2])
    y, _ = layer(x, r)
    y.float().sum().backward()
    assert off(y, reference(layer, x, r)) < 2 * 0.037 and layer.norm_weight.grad.shape == (256,)


def test_no_tokens(ops):
    layer, x, r = make(256, 128, 0)
    y, h = layer(x, r)
    assert y.shape == (0, 128) and h.shape == (0, 256)
    (y.float().sum() + h.float().sum()).backward()
    assert x.grad.shape == (0, 256) and bool((layer.weight.grad == 0).all()) and bool((layer.norm_weight.grad == 0).all())


class Guard:
    """Stands for torch.cuda.device_of: notes for which tensor the current device is switched."""

    def __init__(self, tensor):
        self.tensor = tensor

    def __enter__(self):
        layer8_device.append(self.tensor.device)

    def __exit__(self, *_):
        layer8_device.pop()


def test_launches_go_to_the_operands_device(ops, monkeypatch):
    monkeypatch.setattr(torch.cuda, "device_of", Guard)
    layer, x, r = make()
    y, h = layer(x, r)
    (y.float().sum() + h.float().sum()).backward()
    assert len(ops.devices) == 7 and all(d == x.device for d in ops.devices), list(zip(ops.calls, ops.devices))


def test_only_wanted_gradients_are_computed(ops):
    layer, x, r = make()
    full = {"quant", "norm", "gemmT", "gemmN", "wgrad", "norm_backward"}

    def backward(frozen, loss):
        for name in ("x", "r", "norm_weight", "weight"):
            v = {"x": x, "r": r}.get(name, getattr(layer, name, None))
            v.grad = None
            v.requires_grad_(name not in frozen)
        y, h = layer(x, r)
        ops.calls.clear()
        loss(y.float(), h.float()).backward()
        for name in frozen:
            assert {"x": x, "r": r}.get(name, getattr(layer, name, None)).grad is None
        return set(ops.calls)

    y_loss, h_loss = (lambda y, h: (y * y).sum()), (lambda y, h: (h * h).sum())
    assert backward((), y_loss) == full - {"norm", "gemmT"}
    assert backward(("weight",), y_loss) == {"quant", "gemmN", "norm_backward"}
    assert backward(("x", "r", "norm_weight"), y_loss) == {"wgrad"}
    assert backward((), h_loss) == set()
    h = x.detach() + r.detach()
    assert torch.equal(x.grad, 2 * h) and torch.equal(r.grad, 2 * h) and bool((layer.weight.grad == 0).all()) and bool((layer.norm_weight.grad == 0).all())
