"""A transformer's feed-forward block in 8 bits, from the library's operators:

    h = x + residual,   z = W1 rmsnorm(h) + b1,   y = W2 act(z) + b2 + h

The norm writes e4m3 numbers (b2_rmsnorm_f8); the first product reads them, adds its bias, keeps z for the backward pass and writes act(z) as e4m3 numbers again, the
second one adds its bias and h (both b2_gemm_f8_act).  Backward, the gradient of y is quantised while the second bias's gradient is summed (b2_act_backward), the second weight read along its
other index gives the gradient of z in the same pass (b2_gemm_f8_act with B2_ACT_GRADIENT), and the two 8-bit activations that the forward pass left give the
weights' gradients (b2_wgrad_f8).

Activations are bfloat16 tensors [tokens, features]; sizes are free.  ``python -m paper_1611_08035_b200.ffn8`` trains a small block with AdamW in 8 bits and times
one step of a large one.
"""
from __future__ import annotations

import torch

from . import binding as b2
from .adamw import AdamW
from .capture import AutogradGraphs, GraphWatch, Made, capture_id, capturing, stream_of
from .layer8 import E8, F8, _blocks, _device_of, _Once, _scratch, product, quantise

ACTIVATIONS = {"none": b2.ACT_NONE, "relu": b2.ACT_RELU, "gelu": b2.ACT_GELU, "gelu_tanh": b2.ACT_GELU_TANH, "silu": b2.ACT_SILU}


def _empty8(t: int, d: int, device):
    return torch.empty(t, d, dtype=F8, device=device), torch.empty(t, _blocks(d), dtype=E8, device=device)


def product_act(a, sa, ta, b, sb, m, n, k, act=b2.ACT_NONE, bias=None, z=None, residual=None, c=None, q=None, s=None) -> None:
    """b2_gemm_f8_act of a weight in 128 x 128 blocks, a [m, k] (ta 'T') or [k, m] ('N'), and activations b [n, k], on dense matrices [n, m]."""
    ws = _scratch(b2.b2_gemm_f8_workspace_bytes(ta, "N", m, n, k, a, a.shape[1], b, k), a.device)
    b2.b2_gemm_f8_act(ta, "N", m, n, k, 1.0, a, a.shape[1], sa, sa.shape[1], 128, b, k, sb, sb.shape[1], 1, act, bias, z, m, residual, m, c, m, q, m, s, _blocks(m), ws)


def activation_backward(act, dy, z=None, dz=None, q=None, s=None, db=None) -> None:
    """b2_act_backward of dense matrices [tokens, features]."""
    t, d = dy.shape
    ws = _scratch(b2.b2_act_backward_workspace_bytes(d, t), dy.device) if db is not None else None
    b2.b2_act_backward(d, t, act, dy, d, z, d, dz, d, q, d, s, _blocks(d), db, ws)


class _FeedForward8(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, norm_weight, w1, b1, w2, b2_, quantised, act, eps, keep, graphs):
        (q1, s1), (q2, s2) = quantised
        (t, d), f, device = x.shape, w1.shape[0], x.device
        b1, b2_ = (None if b is None else b.float() for b in (b1, b2_))
        h = torch.empty_like(x) if residual is not None else x
        (nq, ns), (aq, as_) = _empty8(t, d, device), _empty8(t, f, device)
        rstd = torch.empty(t, dtype=torch.float32, device=device) if keep else None
        z = torch.empty(t, f, dtype=torch.bfloat16, device=device) if keep and act != b2.ACT_NONE else None
        y = torch.empty_like(x)
        with _device_of(x):
            b2.b2_rmsnorm_f8(d, t, x, d, residual, d, norm_weight, eps, h if residual is not None else None, d, nq, d, ns, ns.shape[1], rstd)
            product_act(q1, s1, "T", nq, ns, f, t, d, act, b1, z, q=aq, s=as_)
            product_act(q2, s2, "T", aq, as_, d, t, f, b2.ACT_NONE, b2_, residual=h, c=y)
        if keep:
            ctx.save_for_backward(h, norm_weight, rstd, nq, ns, z, aq, as_, q1, s1, q2, s2)
        ctx.act, ctx.has_residual, ctx.graphs, ctx.ran = act, residual is not None, graphs, False
        return y

    @staticmethod
    def backward(ctx, dy):
        if capturing(dy):
            ctx.graphs.refuse(ctx, stream_of(dy))
        ctx.ran = True
        if not torch.is_grad_enabled():
            return _FeedForward8.gradients(ctx, dy)
        with torch.no_grad():  # someone wants to differentiate the gradients: they depend on x and the weights, whatever dy does
            grads = _FeedForward8.gradients(ctx, dy)
        once = iter(_Once.apply(*(g.detach().requires_grad_() for g in grads if g is not None)))
        return tuple(None if g is None else next(once) for g in grads)

    @staticmethod
    def gradients(ctx, dy):
        h, norm_weight, rstd, nq, ns, z, aq, as_, q1, s1, q2, s2 = ctx.saved_tensors
        need_x, need_r, need_norm, need_w1, need_b1, need_w2, need_b2 = ctx.needs_input_grad[:7]
        (t, d), f, device = h.shape, aq.shape[1], h.device
        dy = dy.contiguous()
        f32 = lambda *n: torch.empty(*n, dtype=torch.float32, device=device)  # noqa: E731
        dx = dnw = dw1 = db1 = dw2 = None
        through = need_x or need_r or need_norm or need_w1 or need_b1
        db2 = f32(d) if need_b2 else None

        def weight_gradient(q, s, grad):
            m, n = q.shape[1], grad.shape[1]
            dw = f32(n, m)
            ws = _scratch(b2.b2_wgrad_f8_workspace_bytes(m, n, t, q, m, grad, n), device)
            b2.b2_wgrad_f8(m, n, t, 1.0, q, m, s, s.shape[1], grad, n, 0.0, dw, m, ws)
            return dw

        with _device_of(h):
            dq, ds = _empty8(t, d, device) if through else (None, None)
            if through or need_b2:
                activation_backward(b2.ACT_NONE, dy, q=dq, s=ds, db=db2)
            if need_w2:
                dw2 = weight_gradient(aq, as_, dy)
            if through:
                first = need_x or need_r or need_norm  # whether anything before the first product wants a gradient
                dz = torch.empty(t, f, dtype=torch.bfloat16, device=device) if need_w1 or need_b1 else None
                zq, zs = _empty8(t, f, device) if first else (None, None)
                product_act(q2, s2, "N", dq, ds, f, t, d, ctx.act | b2.ACT_GRADIENT, z=z, c=dz, q=zq, s=zs)
                if need_b1:  # sums of dz as it was stored: half a step of bf16 in each of t terms, to either side; unrounded ones would have to be added up in the product's epilogue
                    db1 = f32(f)
                    activation_backward(b2.ACT_NONE, dz, db=db1)
                if need_w1:
                    dw1 = weight_gradient(nq, ns, dz)
                if first:
                    dnorm = product(q1, s1, 128, "N", zq, zs, 1, d, t, f)
                    dx, dnw = torch.empty_like(h), f32(d)
                    ws = _scratch(b2.b2_rmsnorm_backward_workspace_bytes(d, t), device)
                    b2.b2_rmsnorm_backward(d, t, dnorm, d, h, d, rstd, norm_weight, dy, d, dx, d, dnw, ws)
                    dnw = dnw.to(norm_weight.dtype) if need_norm else None
        return dx if need_x else None, dx if need_r else None, dnw, dw1, db1, dw2, db2, None, None, None, None, None


class FeedForward8(torch.nn.Module):
    """y = block(x, residual).  The weights are kept in float32 for the optimiser and in e4m3 for the products; the 8-bit ones are made anew by the next call after a
    weight was changed in place, replaced, loaded or moved; what changes it unseen by autograd (a replayed CUDA graph) has to call ``requantise()``, which a captured
    training step does itself, first.  It can be differentiated once.

    In a CUDA graph that is captured, an autograd graph of the same block whose backward pass has yet to come must not be alive unless it was made on the capturing stream: such a call is refused.
    So is a captured backward pass that makes the parameters' gradients while any graph of the block that was made on the default stream is alive (they would be made there, which cannot be
    captured)."""

    def __init__(self, features: int, hidden: int, activation: str = "gelu", bias: bool = True, eps: float = 1e-5, device="cuda"):
        super().__init__()
        self.eps, self.act = eps, ACTIVATIONS[activation]
        self.norm_weight = torch.nn.Parameter(torch.ones(features, dtype=torch.bfloat16, device=device))
        self.up = torch.nn.Parameter(torch.randn(hidden, features, device=device) * features**-0.5)
        self.down = torch.nn.Parameter(torch.randn(features, hidden, device=device) * hidden**-0.5)
        self.up_bias = torch.nn.Parameter(torch.zeros(hidden, device=device)) if bias else None
        self.down_bias = torch.nn.Parameter(torch.zeros(features, device=device)) if bias else None
        self._quantised: dict = {}
        self._captured: list = []  # 8-bit weights that captured graphs read, each with a watch of the graph
        self._graphs = AutogradGraphs()

    def __getstate__(self):
        return super().__getstate__() | {"_quantised": {}, "_captured": [], "_graphs": AutogradGraphs()}

    def __setstate__(self, state):  # also one that was saved before there were all of these
        super().__setstate__(state)
        self._quantised, self._captured, self._graphs = {}, [], AutogradGraphs()

    @staticmethod
    def _state(weight):
        return weight, None if weight.is_inference() else weight._version, weight.data_ptr()

    @torch.no_grad()
    def requantise(self) -> None:
        self._let_go()
        weights = {name: getattr(self, name) for name in ("up", "down")}
        pairs = {name: quantise(weight, 128) for name, weight in weights.items()}  # new ones: a backward pass that is still to come reads the old
        made = Made([t for pair in pairs.values() for t in pair], capture_id(self.up) if capturing(self.up) else 0)
        self._quantised = {name: (pairs[name], self._state(weight), made) for name, weight in weights.items()}

    def _let_go(self) -> None:
        """Of what was kept for graphs that are gone."""
        self._captured = [c for c in self._captured if not c[2].gone()]

    def _apply(self, fn, recurse=True):
        self._quantised = {}  # parameters get new storage without a new version
        return super()._apply(fn, recurse)

    def forward(self, x: torch.Tensor, residual: torch.Tensor | None = None):
        d, f = self.up.shape[1], self.up.shape[0]
        # The operators take the extents of x and of the weights for everyone's: what has others would be read beyond its end.
        if x.dim() != 2 or x.shape[1] != d or x.dtype is not torch.bfloat16:
            raise ValueError(f"x is {x.dtype} {tuple(x.shape)}; the block takes bfloat16 [tokens, {d}]")
        if residual is not None and (residual.shape != x.shape or residual.dtype is not x.dtype):
            raise ValueError(f"residual is {residual.dtype} {tuple(residual.shape)}, x {x.dtype} {tuple(x.shape)}: both are alike")
        want = {"norm_weight": (d,), "down": (d, f), "up_bias": (f,), "down_bias": (d,)}
        others = [(n, getattr(self, n)) for n in ("norm_weight", "up", "down", "up_bias", "down_bias")]
        for name, p in others:
            if p is not None and name in want and tuple(p.shape) != want[name]:
                raise ValueError(f"{name} is {tuple(p.shape)}; the block has {d} features and {f} hidden ones: {want[name]}")
        for name, p in (*others, ("residual", residual)):
            if p is not None and p.device != x.device:
                raise ValueError(f"x is on {x.device}, {name} on {p.device}")
        stream = stream_of(x)
        in_capture = capture_id(x) if capturing(x) else 0
        parameters = (self.norm_weight, self.up, self.up_bias, self.down, self.down_bias)
        keep = torch.is_grad_enabled() and any(p is not None and p.requires_grad for p in (x, residual, *parameters))
        if keep and in_capture and not all(node.ran for node in self._graphs.elsewhere(stream)):
            raise RuntimeError("an autograd graph of this block from another stream is alive: delete its results, or make it on the stream that captures")
        for name in ("up", "down"):
            of = self._quantised.get(name)
            now = self._state(getattr(self, name))
            # A tuple's == would compare the parameters' numbers.  What a capture made is there when its graph has run: it is for calls of the same capture.
            if of is None or of[1][0] is not now[0] or of[1][1:] != now[1:] or of[2].capture not in (0, in_capture):
                self.requantise()
                break
        inputs = (x.contiguous(), None if residual is None else residual.contiguous(), self.norm_weight.contiguous(), self.up, self.up_bias, self.down, self.down_bias)
        (up, _, made), (down, _, _) = (self._quantised[n] for n in ("up", "down"))
        made.use(in_capture)
        quantised = (up, down)
        if in_capture and not made.capture:
            self._let_go()
            if not any(c[0] is up and c[2].capture == in_capture for c in self._captured):
                self._captured.append((up, down, GraphWatch(x, in_capture)))
        y = _FeedForward8.apply(*inputs, quantised, self.act, self.eps, keep, self._graphs)
        if keep:
            self._graphs.add(y.grad_fn, stream)
        return y


def train(features: int = 256, hidden: int = 512, tokens: int = 1024, steps: int = 60, lr: float = 3e-3, seed: int = 0, state_bits: int = 8):
    """Losses of a block that learns another one's results with AdamW."""
    torch.manual_seed(seed)
    block, target = FeedForward8(features, hidden), FeedForward8(features, hidden)
    optimiser = AdamW(block.parameters(), lr=lr, betas=(0.9, 0.95), weight_decay=0.0, state_bits=state_bits)
    losses = []
    for _ in range(steps):
        x = torch.randn(tokens, features, device="cuda").bfloat16()
        with torch.no_grad():
            want = target(x)
        loss = (block(x).float() - want.float()).square().mean()
        optimiser.zero_grad()
        loss.backward()
        optimiser.step()
        losses.append(loss.detach())
    return [float(v) for v in losses]


def main() -> None:
    losses = train()
    print(f"loss of a 256 -> 512 -> 256 block over {len(losses)} steps: {losses[0]:.3f} -> {losses[-1]:.4f}")
    t, d, f = 8192, 4096, 16384
    block = FeedForward8(d, f)
    optimiser = AdamW(block.parameters(), lr=1e-4)
    x, r, dy = (torch.randn(t, d, device="cuda").bfloat16() for _ in range(3))
    x.requires_grad_()

    def passes():
        block(x, r).backward(dy)

    def step():
        x.grad = None
        optimiser.zero_grad()
        passes()
        optimiser.step()

    for name, run in (("forward and backward", lambda: (optimiser.zero_grad(), passes())), ("a step with AdamW", step)):
        for _ in range(3):
            run()
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        begin.record()
        for _ in range(10):
            run()
        end.record()
        end.synchronize()
        ms = begin.elapsed_time(end) / 10
        print(f"{name}, {t} tokens, {d} -> {f} -> {d}: {ms:.2f} ms, {12 * t * d * f / ms / 1e9:.0f} TFLOP/s")


if __name__ == "__main__":
    main()
