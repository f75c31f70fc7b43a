"""The 8-bit products at the ends of the scales' range, for outputs as wide as a vocabulary, and in captured graphs."""
import numpy as np
import pytest
import torch

from oracle import f8

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
F8, E8 = torch.float8_e4m3fn, torch.float8_e8m0fnu


def np64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def integers(rows, k, seed):
    return torch.randint(-4, 5, (rows, k), generator=torch.Generator().manual_seed(seed)).float().to(F8)


@pytest.mark.parametrize("scale", [("e8m0", "e8m0"), ("f32", "f32"), ("f32", "e8m0"), ("e8m0", "f32")])
@pytest.mark.parametrize("m,n", [(200, 8), (160, 200), (2304, 2176)])
@pytest.mark.parametrize("byte", [0, 1, 27, 127, 200, 253, 254])
def test_products_under_the_ends_of_e8m0(b2, byte, m, n, scale):
    """A's scales at one end, B's at the other, their products 2^-1 .. 2^1: integers times those are exact (sums of 24 bits and less)."""
    k = 300
    a, b = integers(m, k, byte), integers(n, k, byte + 1)
    g = torch.Generator().manual_seed(byte)
    sa, sb = torch.full((m, 3), byte), (254 - byte + torch.randint(-1, 2, (n, 3), generator=g)).clamp(0, 254)
    to = lambda s, kind: s.to(torch.uint8).cuda().view(E8) if kind == "e8m0" else torch.from_numpy(f8.e8m0(s.numpy()).astype(np.float32)).cuda()  # noqa: E731
    pad = lambda q: torch.nn.functional.pad(q.view(torch.uint8), (0, 4)).cuda().view(F8)  # noqa: E731
    C = torch.empty(n, m, device="cuda")
    b2.b2_gemm_f8("T", "N", m, n, k, 1.0, pad(a), 304, to(sa, scale[0]), 3, 1, pad(b), 304, to(sb, scale[1]), 3, 1, 0.0, C, m)
    want, _ = f8.gemm(np64(a.float()), f8.e8m0(sa.numpy()), 1, np64(b.float()), f8.e8m0(sb.numpy()), 1)
    assert np.array_equal(np64(C), want) and b2.b2_device_status() == 0


@pytest.mark.parametrize("scale", ["e8m0", "f32"])
@pytest.mark.parametrize("out", [BF, F32])
@pytest.mark.parametrize("m,n,k", [(32000, 8, 260), (32000, 1, 128), (40001, 30, 130), (25000, 64, 400), (60000, 16, 128)])
def test_output_layer_of_a_vocabulary(b2, m, n, k, out, scale):
    """More tiles than CTAs at decoding widths: every CTA walks over several.  Integers: the fp32 result is exact, bf16 is its rounding."""
    a, b = integers(m, k, 1), integers(n, k, 2)
    ld = -(-k // 16) * 16
    pad = lambda q: torch.nn.functional.pad(q.view(torch.uint8), (0, ld - k)).cuda().view(F8)  # noqa: E731
    g = torch.Generator().manual_seed(3)
    kb = -(-k // 128)
    sa, sb = torch.randint(126, 129, (-(-m // 128), kb), generator=g), torch.randint(126, 129, (n, kb), generator=g)
    to = lambda s: s.to(torch.uint8).cuda().view(E8) if scale == "e8m0" else torch.exp2(s.float() - 127).cuda()  # noqa: E731
    C = torch.empty(n, m, dtype=out, device="cuda")
    b2.b2_gemm_f8("T", "N", m, n, k, 1.0, pad(a), ld, to(sa), kb, 128, pad(b), ld, to(sb), kb, 1, 0.0, C, m)
    want, _ = f8.gemm(np64(a.float()), f8.e8m0(sa.numpy()), 128, np64(b.float()), f8.e8m0(sb.numpy()), 1)
    assert torch.equal(C.cpu(), torch.from_numpy(want).to(F32).to(out)) and b2.b2_device_status() == 0


def test_captured_graph(b2):
    """Norm, product, a second norm and its gradients captured once and replayed on other inputs: the same bits as the calls give."""
    d, t = 512, 8
    g = torch.Generator().manual_seed(0)
    make = lambda *shape: torch.randn(*shape, generator=g).to(BF).cuda()  # noqa: E731
    x, r, w = make(t, d), make(t, d), torch.ones(d, dtype=BF, device="cuda")
    weight = make(d, d)
    w8, sw = torch.empty(d, d, dtype=F8, device="cuda"), torch.empty(4, 4, dtype=E8, device="cuda")
    b2.b2_quant_f8(d, d, 128, weight, d, w8, d, sw, 4)
    h, q, s, rstd = torch.empty_like(x), torch.empty(t, d, dtype=F8, device="cuda"), torch.empty(t, 4, dtype=E8, device="cuda"), torch.empty(t, device="cuda")
    y, dx, dw, grad = torch.empty_like(x), torch.empty_like(x), torch.empty(d, device="cuda"), torch.empty(d, d, device="cuda")
    ws = torch.empty(b2.b2_rmsnorm_backward_workspace_bytes(d, t), dtype=torch.uint8, device="cuda")

    def step():
        for _ in range(3):
            b2.b2_rmsnorm_f8(d, t, x, d, r, d, w, 1e-5, h, d, q, d, s, 4, rstd)
            b2.b2_gemm_f8("T", "N", d, t, d, 1.0, w8, d, sw, 4, 128, q, d, s, 4, 1, 0.0, y, d)
            b2.b2_rmsnorm_backward(d, t, y, d, h, d, rstd, w, r, d, dx, d, dw, ws)
            b2.b2_wgrad_f8(d, d, t, 1.0, q, d, s, 4, y, d, 0.0, grad, d)
            x.copy_(dx)

    outputs = (h, q.view(torch.uint8), s.view(torch.uint8), rstd, y, dx, dw, grad)
    start = [(make(t, d), make(t, d)) for _ in range(2)]
    wants = []
    for xs, rs in start:
        x.copy_(xs), r.copy_(rs)
        step()
        wants.append([v.clone() for v in outputs])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for (xs, rs), want in zip(start, wants):
        x.copy_(xs), r.copy_(rs)
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(outputs, want))
    assert b2.b2_device_status() == 0


def test_layer_of_no_tokens(b2):
    from paper_1611_08035_b200 import layer8
    layer = layer8.NormLinear8(256, 128)
    x, r = (torch.empty(0, 256, dtype=BF, device="cuda").requires_grad_() for _ in range(2))
    y, h = layer(x, r)
    (y.float().sum() + h.float().sum()).backward()
    assert y.shape == (0, 128) and x.grad.shape == (0, 256) and b2.b2_device_status() == 0
    assert bool((layer.weight.grad == 0).all()) and bool((layer.norm_weight.grad == 0).all())


def test_layer_after_its_weight_was_loaded(b2):
    """The same bits as a layer that was made with that weight, also on a stream of the caller's."""
    from paper_1611_08035_b200 import layer8
    torch.manual_seed(1)
    a, b = layer8.NormLinear8(384, 200), layer8.NormLinear8(384, 200)
    x = torch.randn(7, 384, device="cuda").to(BF)
    want, _ = a(x)
    b.load_state_dict(a.state_dict())
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        got, _ = b(x)
    stream.synchronize()
    assert torch.equal(got, want) and not torch.equal(a(x)[0], layer8.NormLinear8(384, 200)(x)[0])
