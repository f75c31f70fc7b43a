"""The feed-forward block and the AdamW optimiser around the operators.

The block against the same one in fp32 autograd.  What differs are the roundings to e4m3 (2.6 % of a number in the mean square, spread evenly over a step; 3.7 % for a product of
two such operands, see test_layer8_gpu.py) and bf16 ones (0.2 %).  y - h: norm and first weight 3.7 %, that result's own rounding and the second weight's 3.7 % more: 5.3 % of its norm, as no activation here
stretches an error by more than 1.13: 6 %.  Second weight's gradient: its activation is off by 3.7 % (times 1.13) and 2.6 %: 5 %.  Gradient of z: gradient of y and second weight 3.7 %, slope
at a z that is off by 3.7 %: slopes change by at most 0.8 for z changed by 1, and |z| is about 1: 3 % more: 4.8 %; first weight's gradient with the norm's 2.6 %: 5.5 %; gradient of x with two
more roundings 6.1 %.  Twice that is allowed.  relu's slope is a step: a z that is off by 3.7 % of its spread changes its sign with probability atan(0.037) / pi = 1.18 %, and then the gradient of z, half of
whose numbers are not 0, is wrong altogether: sqrt(1.18 % / 50 %) = 15.3 % of its norm, independent of the other errors."""
import copy

import pytest
import torch

from paper_1611_08035_b200 import ffn8
from paper_1611_08035_b200.adamw import AdamW

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def reference(block, x, r, dy, act):
    p = {n: v.detach().float().requires_grad_() for n, v in block.named_parameters()}
    x, r = (None if v is None else v.detach().float().requires_grad_() for v in (x, r))
    h = x if r is None else x + r
    n = h * torch.rsqrt(h.square().mean(1, keepdim=True) + block.eps) * p["norm_weight"]
    z = n @ p["up"].t() + p.get("up_bias", 0.0)
    f = {"none": lambda v: v, "relu": torch.relu, "gelu": torch.nn.functional.gelu, "gelu_tanh": lambda v: torch.nn.functional.gelu(v, approximate="tanh"), "silu": torch.nn.functional.silu}
    y = f[act](z) @ p["down"].t() + p.get("down_bias", 0.0)
    (y + h).backward(dy.float())
    return y.detach(), {"x": x.grad, **({"r": r.grad} if r is not None else {}), **{k: v.grad for k, v in p.items()}}


def off(a, b):
    return float((a.detach().float() - b).norm() / b.norm())


@pytest.mark.parametrize("t,d,f,act,bias,residual", [(300, 512, 768, "gelu", True, True), (33, 1003, 257, "silu", True, False), (1, 128, 128, "gelu_tanh", False, True),
                                                    (1600, 384, 1700, "gelu", True, True), (70, 256, 512, "relu", False, False), (40, 130, 300, "none", True, True)])
def test_block_and_gradients(b2, t, d, f, act, bias, residual):
    torch.manual_seed(t)
    block = ffn8.FeedForward8(d, f, act, bias)
    with torch.no_grad():
        block.norm_weight += 0.1 * torch.randn(d, device="cuda").bfloat16()
        for b in (block.up_bias, block.down_bias):
            if b is not None:
                b += 0.3 * torch.randn_like(b)
    x, r = (torch.randn(t, d, device="cuda").bfloat16().requires_grad_() for _ in range(2))
    r = r if residual else None
    dy = torch.randn(t, d, device="cuda").bfloat16()
    y = block(x, r)
    y.backward(dy)
    assert b2.b2_device_status() == 0
    want, grads = reference(block, x, r, dy, act)
    h = x.float() + (0 if r is None else r.float())
    assert off(y.float() - h, want) < 2 * 0.06
    got = {"x": x.grad, **({"r": r.grad} if r is not None else {}), **{k: v.grad for k, v in block.named_parameters()}}
    step = 0.153 if act == "relu" else 0.0
    with_step = lambda e: 2 * (e * e + step * step) ** 0.5  # noqa: E731
    # x also gets dy itself, which is exact: what the block adds is what is judged
    for k in ("x", "r"):
        if k in grads:
            assert off(got.pop(k).float() - dy.float(), grads.pop(k) - dy.float()) < with_step(0.061), k
    bounds = {"norm_weight": 0.061, "up": 0.055, "down": 0.05, "up_bias": 0.048, "down_bias": 2.0**-9}
    for k, v in grads.items():
        assert off(got[k], v) < (2 * bounds[k] if k.startswith("down") else with_step(bounds[k])), k


def test_only_wanted_gradients(b2):
    block = ffn8.FeedForward8(256, 300)
    x, dy = torch.randn(20, 256, device="cuda").bfloat16(), torch.randn(20, 256, device="cuda").bfloat16()
    block(x).backward(dy)
    every = {n: p.grad for n, p in block.named_parameters()}
    for names in (("down",), ("down_bias",), ("up",), ("up_bias",), ("norm_weight",), ("up", "down_bias"), ()):
        for n, p in block.named_parameters():
            p.grad = None
            p.requires_grad_(n in names)
        xx = x.clone().requires_grad_(not names)
        block(xx).backward(dy)
        for n, p in block.named_parameters():
            assert (p.grad is None) == (n not in names) and (p.grad is None or torch.equal(p.grad, every[n])), (names, n)
        assert (xx.grad is None) == bool(names)
    for p in block.parameters():
        p.requires_grad_(True)
    with torch.no_grad():
        a = block(x)
    assert torch.equal(a, block(x)) and not a.requires_grad


def test_refusals_and_no_tokens(b2):
    block = ffn8.FeedForward8(256, 300)
    for bad in (torch.zeros(3, 255, device="cuda", dtype=BF), torch.zeros(3, 256, device="cuda"), torch.zeros(256, device="cuda", dtype=BF), torch.zeros(3, 256, dtype=BF)):
        with pytest.raises(ValueError):
            block(bad)
    x = torch.zeros(3, 256, device="cuda", dtype=BF)
    with pytest.raises(ValueError):
        block(x, torch.zeros(2, 256, device="cuda", dtype=BF))
    with pytest.raises(KeyError):
        ffn8.FeedForward8(256, 300, "tanh")
    empty = torch.zeros(0, 256, device="cuda", dtype=BF, requires_grad=True)
    block(empty).sum().backward()
    assert empty.grad.shape == (0, 256) and all(bool((p.grad == 0).all()) for p in block.parameters())
    xx = torch.randn(3, 256, device="cuda").bfloat16().requires_grad_()
    grad, = torch.autograd.grad(block(xx).float().square().sum(), xx, create_graph=True)
    with pytest.raises(RuntimeError, match="once"):
        grad.float().sum().backward()


def test_weights_that_changed(b2):
    """The 8-bit weights follow changes in place, the optimiser's among them; a backward pass uses those of its forward pass."""
    block = ffn8.FeedForward8(256, 384)
    x = torch.randn(30, 256, device="cuda").bfloat16()
    before = block(x)
    with torch.no_grad():
        block.up *= 2.0
    after = block(x)
    assert not torch.equal(before, after)
    want = copy.deepcopy(block)
    assert torch.equal(after, want(x))
    optimiser = AdamW(block.parameters(), lr=1e-2)
    y = block(x.requires_grad_())
    y.sum().backward(retain_graph=True)
    first = x.grad.clone()
    with torch.no_grad():
        block.up *= 0.5
        assert not torch.equal(block(x), after)
    x.grad = None
    y.sum().backward(retain_graph=True)
    assert torch.equal(x.grad, first)
    after = block(x).detach()
    optimiser.step()
    assert not torch.equal(block(x), after)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):  # the norm's weight is not what it was
        y.sum().backward()
    fresh = ffn8.FeedForward8(256, 384)
    fresh.load_state_dict(block.state_dict())
    assert torch.equal(fresh(x), block(x))


# ---- the optimiser ------------------------------------------------------------------------------------------------------
def twin(sizes, seed=0, dtype=F32):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.nn.Parameter((0.1 * torch.randn(s, device="cuda", generator=g)).to(dtype)) for s in sizes]


SIZES = [(300, 130), (7,), (64, 128), (5000,), ()]


def test_32_bits_is_adamw(b2):
    """20 steps beside torch's.  Both make a dozen fp32 roundings of a step (lr 1e-2, at most 1.3 of it) and one of p in each of 20 steps."""
    a, b = twin(SIZES), twin(SIZES)
    ours, theirs = (c(p, lr=1e-2, betas=(0.9, 0.99), weight_decay=0.1, **kw) for c, p, kw in ((AdamW, a, {"state_bits": 32}), (torch.optim.AdamW, b, {"foreach": False})))
    g = torch.Generator(device="cuda").manual_seed(1)
    for _ in range(20):
        for p, q in zip(a, b):
            p.grad = torch.randn(p.shape, device="cuda", generator=g)
            q.grad = p.grad.clone()
        ours.step(), theirs.step()
    for p, q in zip(a, b):
        assert float((p - q).detach().abs().max()) <= 20 * 2.0**-24 * (float(q.detach().abs().max()) * 2 + 16 * 1.3e-2)


@pytest.mark.parametrize("dtype", [F32, BF])
def test_8_bits_stays_near(b2, dtype):
    """One step from nothing is the 32-bit step to a rounding; after more, moments are off by an e4m3 step (1/8) at most and steps by as much."""
    a, b = twin([(300, 130)], dtype=dtype), twin([(300, 130)], dtype=dtype)
    eight, full = AdamW(a, lr=1e-2, state_bits=8), AdamW(b, lr=1e-2, state_bits=32)
    g = torch.Generator(device="cuda").manual_seed(1)
    start = a[0].detach().float().clone()
    for i in range(3):
        a[0].grad = torch.randn(300, 130, device="cuda", generator=g).to(dtype)
        b[0].grad = a[0].grad.clone()
        eight.step(), full.step()
        if i == 0:
            assert float((a[0] - b[0]).detach().float().abs().max()) <= (2.0**-8 if dtype is BF else 2.0**-22) * float(a[0].detach().abs().max())
    assert eight.state[a[0]]["m"].dtype is torch.float8_e4m3fn and eight.state[a[0]]["sm"].numel() == (300 * 130 + 127) // 128
    moved = (a[0].detach().float() - start) - (b[0].detach().float() - start)
    assert float(moved.norm()) <= 0.3 * float((b[0].detach().float() - start).norm())


def test_states_are_saved_and_loaded(b2):
    a = twin(SIZES)
    opt = AdamW(a, lr=1e-2)
    g = torch.Generator(device="cuda").manual_seed(1)
    grads = [[torch.randn(p.shape, device="cuda", generator=g) for p in a] for _ in range(4)]

    def go(opt, params, some):
        for gs in some:
            for p, x in zip(params, gs):
                p.grad = x.clone()
            opt.step()

    go(opt, a, grads[:2])
    saved, at = copy.deepcopy(opt.state_dict()), [p.detach().clone() for p in a]
    go(opt, a, grads[2:])
    b = [torch.nn.Parameter(x) for x in at]
    other = AdamW(b, lr=1e-2)
    other.load_state_dict(saved)
    go(other, b, grads[2:])
    assert all(torch.equal(p, q) for p, q in zip(a, b))
    assert other.state[b[0]]["m"].dtype is torch.float8_e4m3fn and other.state[b[1]]["m"].dtype is F32


def test_optimiser_refusals(b2):
    with pytest.raises(ValueError):
        AdamW(twin([(3,)]), state_bits=16)
    with pytest.raises(ValueError):
        AdamW([torch.nn.Parameter(torch.zeros(4, 6, device="cuda").t())])
    with pytest.raises(ValueError):
        AdamW([torch.nn.Parameter(torch.zeros(4, device="cuda", dtype=torch.float64))])
    p = torch.nn.Parameter(torch.zeros(8))
    p.grad = torch.ones(8)
    with pytest.raises(TypeError):  # a host tensor
        AdamW([p]).step()
    q, = twin([(40, 3)])
    q.grad = torch.randn(3, 40, device="cuda").t()  # not contiguous: taken as it is
    w, = twin([(40, 3)])
    w.grad = q.grad.contiguous()
    AdamW([q]).step(), AdamW([w]).step()
    assert torch.equal(q, w)


def test_training_step_captured(b2):
    """Forward, backward, clipping and step in a replayed graph: the same bits as step by step."""
    def make():
        torch.manual_seed(5)
        block = ffn8.FeedForward8(256, 512)
        return block, AdamW(block.parameters(), lr=3e-3, betas=(0.9, 0.95), capturable=True, least_8bit=256)

    def one(block, opt, x, dy):
        block.requantise()
        block(x).backward(dy)
        norm = torch.stack([p.grad.float().norm() for p in block.parameters()]).norm()
        opt.step(grad_scale=(1.0 / norm.clamp(min=1.0)).reshape(1))
        opt.zero_grad()

    data = [(torch.randn(70, 256, device="cuda").bfloat16(), torch.randn(70, 256, device="cuda").bfloat16()) for _ in range(5)]
    eager, opt = make()
    for x, dy in data:
        one(eager, opt, x, dy)
    block, opt = make()
    x, dy = (v.clone() for v in data[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):  # the first step, on the stream where the leaves' gradients will be captured
        one(block, opt, x, dy)
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=side):
            one(block, opt, x, dy)
    for a, b in data[1:]:
        x.copy_(a), dy.copy_(b)
        graph.replay()
    torch.cuda.synchronize()
    for p, q in zip(eager.parameters(), block.parameters()):
        assert torch.equal(p, q)
    assert b2.b2_device_status() == 0


def test_captures_and_eager_calls_side_by_side(b2):
    """A captured call keeps the 8-bit weights that it reads, one that makes its own leaves eager calls theirs, and one beside a living eager graph is refused."""
    torch.manual_seed(6)
    block = ffn8.FeedForward8(256, 512)
    x = torch.randn(40, 256, device="cuda").bfloat16()
    with torch.no_grad():
        want = block(x)
        graph, own = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            y = block(x)
        with torch.cuda.graph(own):
            block.requantise()
            z = block(x)
        assert torch.equal(block(x), want)  # before either graph has run
        block.up.mul_(2.0)
        changed = block(x)
        filler = [torch.full((512 * 256,), 255, dtype=torch.uint8, device="cuda") for _ in range(8)]  # where freed weights were
        graph.replay(), own.replay()
        assert torch.equal(y, want) and torch.equal(z, changed) and not torch.equal(want, changed)
        del filler
    alive = block(x)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with pytest.raises(RuntimeError, match="alive"):
        with torch.cuda.graph(graph):
            block(x)
    alive.sum().backward()
    optimiser = AdamW(block.parameters())
    optimiser.step()
    torch.cuda.synchronize()
    with pytest.raises(RuntimeError, match="capturable"):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            optimiser.step()
    torch.cuda.synchronize()
    assert b2.b2_device_status() == 0


def test_training_runs(b2):
    for bits in (8, 32):
        losses = ffn8.train(steps=3, state_bits=bits)
        assert len(losses) == 3 and all(v == v for v in losses)
