"""The 8-bit layer (norm, product, their gradients) against the same layer in fp32 autograd.

What differs are the roundings to e4m3: of the norm's result, the weight and the output's gradient.  One rounding is off by at
most 2^-4 of a number and, spread evenly over a step, by 2^-4 / sqrt(3) / 1.4 = 2.6 % in the mean square; block scales leave no number further from
its block's largest than 2^-9 of it unrounded.  A product of two such operands is off by sqrt(2) * 2.6 % = 3.7 % of its norm (errors of
different numbers are independent), one with a single such operand by 2.6 %; twice that is allowed."""
import pytest
import torch

from paper_1611_08035_b200 import layer8

pytestmark = pytest.mark.gpu


def reference(x, r, nw, w, eps, dy, dh):
    x, r, nw, w = (v.detach().float().requires_grad_() for v in (x, r, nw, w))
    h = x + r
    y = h * torch.rsqrt(h.square().mean(1, keepdim=True) + eps) * nw @ w.t()
    torch.autograd.backward([y, h], [dy.float(), dh.float()])
    return y.detach(), h.detach(), x.grad, r.grad, nw.grad, w.grad


@pytest.mark.parametrize("t,d,n", [(300, 512, 384), (33, 1003, 257), (1, 128, 128)])
def test_layer_and_gradients(b2, t, d, n):
    torch.manual_seed(t)
    layer = layer8.NormLinear8(d, n)
    with torch.no_grad():
        layer.norm_weight += 0.1 * torch.randn(d, device="cuda").bfloat16()
    x, r = (torch.randn(t, d, device="cuda").bfloat16().requires_grad_() for _ in range(2))
    dy, dh = torch.randn(t, n, device="cuda").bfloat16(), torch.randn(t, d, device="cuda").bfloat16()
    y, h = layer(x, r)
    torch.autograd.backward([y, h], [dy, dh])
    assert b2.b2_device_status() == 0
    want = reference(x, r, layer.norm_weight, layer.weight, layer.eps, dy, dh)
    off = lambda a, b: float((a.detach().float() - b).norm() / b.norm())  # noqa: E731
    assert off(h, want[1]) < 2.0**-8
    assert off(y, want[0]) < 2 * 0.037
    assert off(x.grad, want[2]) < 2 * 0.037 and torch.equal(x.grad, r.grad)
    assert off(layer.norm_weight.grad, want[4]) < 2 * 0.037
    assert off(layer.weight.grad, want[5]) < 2 * 0.026


def test_without_residual(b2):
    layer = layer8.NormLinear8(256, 128)
    x = torch.randn(5, 256, device="cuda").bfloat16().requires_grad_()
    y, h = layer(x)
    y.sum().backward()
    assert torch.equal(h, x) and bool(torch.isfinite(x.grad).all()) and y.shape == (5, 128)


def test_gradient_of_h_alone(b2):
    layer = layer8.NormLinear8(256, 128)
    x, r = (torch.randn(5, 256, device="cuda").bfloat16().requires_grad_() for _ in range(2))
    _, h = layer(x, r)
    h.backward(torch.full_like(h, 0.5))
    assert bool((x.grad == 0.5).all()) and bool((layer.weight.grad == 0).all())


def test_training_learns(b2):
    losses = layer8.train(steps=40)
    assert losses[0] > 1.5 and losses[-1] < 0.05 * losses[0]
