"""A transformer block's norm and linear layer in 8 bits, from the library's operators:

    h = x + residual,   y = rmsnorm(h) W^T

The norm writes its result as e4m3 numbers with a scale for each 128 features (b2_rmsnorm_f8).  The product reads them as they
are (b2_gemm_f8, against weights in 128 x 128 blocks), and so does the backward pass: the same 8-bit activation, kept
instead of a 16-bit one, gives the weight gradient (b2_wgrad_f8), the same 8-bit weight read along its other index the
gradient of the norm's result, and b2_rmsnorm_backward the gradients of x, the residual and the norm's weight.

Activations are bfloat16 tensors [tokens, features]; sizes are free.  ``python -m paper_1611_08035_b200.layer8`` trains a small
layer towards a target and times one step of a large one.
"""
from __future__ import annotations

import contextlib

import torch

from . import binding as b2
from .capture import AutogradGraphs, GraphWatch, Made, capture_id, capturing, stream_of

F8, E8 = torch.float8_e4m3fn, torch.float8_e8m0fnu


def _blocks(n: int) -> int:
    return (n + 127) // 128


def _scratch(nbytes: int, device) -> torch.Tensor | None:
    return torch.empty(nbytes, dtype=torch.uint8, device=device) if nbytes else None


_HERE = contextlib.nullcontext()


def _device_of(x):
    """Makes x's device the current one, to a stream of which the calls go; costs nothing where it is (switching there and back takes 1.5 us)."""
    return _HERE if x.is_cuda and x.get_device() == torch._C._cuda_getDevice() else torch.cuda.device_of(x)


def quantise(x: torch.Tensor, block: int = 1):
    """x [rows, features] (bfloat16 or float32) as e4m3 numbers and the e8m0 scales of its block x 128 tiles."""
    x = x.contiguous()
    t, d = x.shape
    q = torch.empty(t, d, dtype=F8, device=x.device)
    s = torch.empty((t + block - 1) // block, _blocks(d), dtype=E8, device=x.device)
    with _device_of(x):
        b2.b2_quant_f8(d, t, block, x, d, q, d, s, s.shape[1])
    return q, s


def product(a, sa, block_a, ta, b, sb, block_b, m, n, k, out_dtype=torch.bfloat16):
    """[n, m] = B A^T of block-scaled operands: b [n, k]; a [m, k] (ta 'T') or [k, m] (ta 'N')."""
    c = torch.empty(n, m, dtype=out_dtype, device=a.device)
    ws = _scratch(b2.b2_gemm_f8_workspace_bytes(ta, "N", m, n, k, a, a.shape[1], b, k), a.device)
    with _device_of(a):
        b2.b2_gemm_f8(ta, "N", m, n, k, 1.0, a, a.shape[1], sa, sa.shape[1], block_a, b, k, sb, sb.shape[1], block_b, 0.0, c, m, ws)
    return c


class _Once(torch.autograd.Function):
    """Gradients as they are, which cannot be differentiated again."""

    @staticmethod
    def forward(ctx, *grads):
        return tuple(g.view_as(g) for g in grads)

    @staticmethod
    def backward(ctx, *_):
        raise RuntimeError("the 8-bit layer's gradients have no gradient of their own: it can be differentiated once")


class _NormLinear8(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, norm_weight, weight, w8, sw, eps, graphs):
        ctx.set_materialize_grads(False)  # no gradient for h: nothing to add
        t, d = x.shape
        n = weight.shape[0]
        h = torch.empty_like(x) if residual is not None else x
        q, s = torch.empty(t, d, dtype=F8, device=x.device), torch.empty(t, _blocks(d), dtype=E8, device=x.device)
        rstd = torch.empty(t, dtype=torch.float32, device=x.device)
        with _device_of(x):
            b2.b2_rmsnorm_f8(d, t, x, d, residual, d, norm_weight, eps, h if residual is not None else None, d, q, d, s, s.shape[1], rstd)
        y = product(w8, sw, 128, "T", q, s, 1, n, t, d)
        ctx.save_for_backward(h, norm_weight, q, s, rstd, w8, sw)
        ctx.has_residual, ctx.graphs = residual is not None, graphs
        return y, h

    @staticmethod
    def backward(ctx, dy, dh):
        given = dh if dy is None else dy
        if given is not None and capturing(given):
            ctx.graphs.refuse(ctx, stream_of(given))
        if not torch.is_grad_enabled():
            return _NormLinear8.gradients(ctx, dy, dh)
        with torch.no_grad():  # someone wants to differentiate the gradients: they depend on x and the weights, whatever dy does
            grads = _NormLinear8.gradients(ctx, dy, dh)
        once = iter(_Once.apply(*(g.detach().requires_grad_() for g in grads if g is not None)))
        return tuple(None if g is None else next(once) for g in grads)

    @staticmethod
    def gradients(ctx, dy, dh):
        h, norm_weight, q, s, rstd, w8, sw = ctx.saved_tensors
        wants_x, wants_residual, wants_norm, wants_weight = ctx.needs_input_grad[:4]
        (t, d), n, device = h.shape, w8.shape[0], h.device
        dx = dnw = dweight = None
        if dy is None:  # a loss on h alone, which the norm and the product do not touch
            if wants_norm:
                dnw = torch.zeros_like(norm_weight)
            if wants_weight:
                dweight = torch.zeros(n, d, dtype=torch.float32, device=device)
            return dh, dh if ctx.has_residual else None, dnw, dweight, None, None, None, None
        dy = dy.contiguous()
        with _device_of(h):
            if wants_x or wants_residual or wants_norm:
                dq, ds = quantise(dy)
                dnorm = product(w8, sw, 128, "N", dq, ds, 1, d, t, n)
            if wants_weight:
                dweight = torch.empty(n, d, dtype=torch.float32, device=device)
                ws = _scratch(b2.b2_wgrad_f8_workspace_bytes(d, n, t, q, d, dy, n), device)
                b2.b2_wgrad_f8(d, n, t, 1.0, q, d, s, s.shape[1], dy, n, 0.0, dweight, d, ws)
            if wants_x or wants_residual or wants_norm:
                dx, dnw = torch.empty_like(h), torch.empty(d, dtype=torch.float32, device=device)
                ws = _scratch(b2.b2_rmsnorm_backward_workspace_bytes(d, t), device)
                b2.b2_rmsnorm_backward(d, t, dnorm, d, h, d, rstd, norm_weight, None if dh is None else dh.contiguous(), d, dx, d, dnw, ws)
                dnw = dnw.to(norm_weight.dtype) if wants_norm else None
        return dx, dx if ctx.has_residual else None, dnw, dweight, None, None, None, None


class NormLinear8(torch.nn.Module):
    """y, h = layer(x, residual): h = x + residual (x without one), y = rmsnorm(h) W^T.  W is kept in float32 for the optimiser
    and in e4m3 for the products.  The 8-bit one is made anew by the next call after the weight was changed in place, replaced, loaded or
    moved; what changes it unseen by autograd (through ``weight.data``, or in a replayed CUDA graph) has to call ``requantise()``.  What a captured graph reads of it is kept while the
    graph lives, and what one makes of it is read by calls of the same capture alone.

    While a backward pass is captured that makes the parameters' gradients, no autograd graph of the same layer that was made on the default stream may be alive (they would be
    made there, which cannot be captured): such a pass is refused."""

    def __init__(self, features: int, outputs: int, eps: float = 1e-5, device="cuda"):
        super().__init__()
        self.eps = eps
        self.norm_weight = torch.nn.Parameter(torch.ones(features, dtype=torch.bfloat16, device=device))
        self.weight = torch.nn.Parameter(torch.randn(outputs, features, device=device) * features**-0.5)
        self._quantised = None
        self._captured: list = []  # 8-bit weights that captured graphs read, each with a watch of the graph
        self._graphs = AutogradGraphs()
        if self.weight.is_cuda:
            self.requantise()

    @staticmethod
    def _state(weight):
        """The parameter and the number of changes that it has seen (a tuple: as an attribute of its own it would count as a second parameter)."""
        return weight, None if weight.is_inference() else weight._version

    @torch.no_grad()
    def requantise(self) -> None:
        self._let_go()
        self.w8, self.sw = pair = quantise(self.weight, 128)
        self._quantised = (*self._state(self.weight), Made(pair, capture_id(self.weight) if capturing(self.weight) else 0))

    def __getstate__(self):
        return super().__getstate__() | {"_quantised": None, "_captured": [], "_graphs": AutogradGraphs()}

    def __setstate__(self, state):  # also one that was saved before there were all of these
        super().__setstate__(state)
        self._quantised, self._captured, self._graphs = None, [], AutogradGraphs()

    def _let_go(self) -> None:
        """Of what was kept for graphs that are gone."""
        self._captured = [c for c in self._captured if not c[1].gone()]

    def _apply(self, fn, recurse=True):
        self._quantised = None  # parameters get new storage without a new version
        return super()._apply(fn, recurse)

    def forward(self, x: torch.Tensor, residual: torch.Tensor | None = None):
        weight, norm_weight = self.weight, self.norm_weight
        # The operators take the extents of x and of the weight for everyone's: what has others would be read beyond its end.
        shape, d, device = x.shape, weight.shape[1], x.device
        if len(shape) != 2 or shape[1] != d:
            raise ValueError(f"x is {tuple(shape)}; the layer takes [tokens, {d}]")
        if residual is not None and residual.shape != shape:
            raise ValueError(f"residual is {tuple(residual.shape)}, x {tuple(shape)}: both have one shape")
        if norm_weight.shape != (d,):
            raise ValueError(f"norm_weight is {tuple(norm_weight.shape)}; the weight has {d} features")
        if weight.device != device or norm_weight.device != device or (residual is not None and residual.device != device):
            raise ValueError(f"x is on {device}, the weight on {weight.device}, the norm's on {norm_weight.device}, the residual on {None if residual is None else residual.device}")
        of, in_capture = self._quantised, capture_id(x) if capturing(x) else 0
        # What a capture made is there when its graph has run: it is for calls of the same capture.
        if of is None or of[0] is not weight or of[1] != self._state(weight)[1] or of[2].capture not in (0, in_capture):
            self.requantise()
        made = self._quantised[2]
        made.use(in_capture)
        if in_capture and not made.capture:
            self._let_go()
            if not any(c[0] is made.tensors and c[1].capture == in_capture for c in self._captured):
                self._captured.append((made.tensors, GraphWatch(x, in_capture)))
        y, h = _NormLinear8.apply(x.contiguous(), None if residual is None else residual.contiguous(), norm_weight.contiguous(), weight, *made.tensors, self.eps, self._graphs)
        if y.grad_fn is not None:
            self._graphs.add(y.grad_fn, stream_of(x))
        return y, h


def train(features: int = 512, outputs: int = 384, tokens: int = 1024, steps: int = 40, lr: float = 0.5, seed: int = 0):
    """Losses of a layer that learns another one's results by gradient descent."""
    torch.manual_seed(seed)
    layer = NormLinear8(features, outputs)
    target = torch.randn(outputs, features, device="cuda") * features**-0.5
    losses = []
    for _ in range(steps):
        x, r = (torch.randn(tokens, features, device="cuda").bfloat16() for _ in range(2))
        h = (x + r).float()
        want = (h * torch.rsqrt(h.square().mean(1, keepdim=True) + layer.eps)) @ target.t()
        y, _ = layer(x, r)
        loss = (y.float() - want).square().mean()
        loss.backward()
        with torch.no_grad():
            layer.weight -= lr * outputs * layer.weight.grad
            layer.weight.grad = layer.norm_weight.grad = None
        layer.requantise()
        losses.append(loss.detach())
    return [float(v) for v in losses]


def main() -> None:
    losses = train()
    print(f"loss of a 512 -> 384 layer over {len(losses)} steps: {losses[0]:.3f} -> {losses[-1]:.4f}")
    t, d = 8192, 8192
    layer = NormLinear8(d, d)
    x, r, dy = (torch.randn(t, d, device="cuda").bfloat16() for _ in range(3))
    x.requires_grad_()

    def step():
        y, _ = layer(x, r)
        y.backward(dy)
        x.grad = layer.weight.grad = layer.norm_weight.grad = None

    for _ in range(3):
        step()
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    begin.record()
    for _ in range(10):
        step()
    end.record()
    end.synchronize()
    ms = begin.elapsed_time(end) / 10
    print(f"forward and backward, {t} tokens, {d} -> {d}: {ms:.2f} ms, {6 * t * d * d / ms / 1e9:.0f} TFLOP/s")


if __name__ == "__main__":
    main()
