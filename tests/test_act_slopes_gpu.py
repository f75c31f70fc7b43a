"""gelu's derivative where it is small: Phi(z) + z phi(z) = -exp(-z^2/2) (x c + h) for z = -x, c = 1/sqrt(2 pi), h = -Phi(-x) exp(x^2/2).

Tolerance, u = 2^-24, derived before the first run, for 1 <= x <= 13 (beyond 13.2 the exponential is subnormal): the exponent x^2 log2(e)/2 is made of a rounded constant and two rounded
products, 2.5 u of itself, which is x^2/2 in nats: 1.25 x^2 u of the exponential, whose own approximation is within 2^-22 = 4 u; h: its polynomial 3 u and eight steps' roundings, 1/(1 + 0.3 x) 2 u: 14 u
of h, and c x and the sum one each; |h| / (c x + h) <= 1.91 at x = 1 and falls, c x / (c x + h) <= 2.91: 1.91 * 14 + 2.91 + 1 < 31 u; the last product 1 u: (1.25 x^2 + 36) u.  For
z > 0 the result is 1 and more, for -1 < z within 2^-18 of the definition as everywhere.  What is multiplied is stored in fp32 (u)."""
import numpy as np
import pytest
import torch

from oracle import ffn

pytestmark = pytest.mark.gpu
U = 2.0**-24
F8, E8 = torch.float8_e4m3fn, torch.float8_e8m0fnu


def np64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def allowed(z, slope):
    return np.where(z <= -1, (1.25 * z * z + 38) * U * np.abs(slope), 2.0**-18)


def negative(n, d, seed):
    g = torch.Generator().manual_seed(seed)
    return 14.0 * torch.rand(n, d, generator=g) - 13.0  # -13 .. 1


@pytest.mark.parametrize("pad", [0, 1])
def test_backward_pass(b2, pad):
    d, t = 1000, 300
    ld = d + pad
    z = torch.zeros(t, ld)
    z[:, :d] = negative(t, d, 1)
    dz = torch.empty(t, ld, device="cuda")
    b2.b2_act_backward(d, t, b2.ACT_GELU, torch.ones(t, ld, device="cuda"), ld, z.cuda(), ld, dz, ld, None, d, None, 8, None)
    z = np64(z[:, :d])
    want = ffn.act_slope(z, "gelu")
    off = np.abs(np64(dz[:, :d]) - want) / allowed(z, want)
    assert off.max() <= 1, (off.max(), z.flat[off.argmax()])


@pytest.mark.parametrize("m,n,k,pad", [(300, 7, 128, 0), (512, 20, 4096, 0), (300, 200, 256, 0), (301, 203, 128, 0), (512, 500, 2048, 0), (1600, 1504, 128, 0), (1600, 1504, 128, 1)])
def test_gradient_form(b2, m, n, k, pad):
    """Sums of a single product: 64 whatever else; decoding, tiles of one CTA, splits, pairs of CTAs, columns that start anywhere."""
    ld = m + pad
    a, b = torch.zeros(m, k, device="cuda"), torch.zeros(n, k, device="cuda")
    a[:, 5], b[:, 5] = 8.0, 8.0
    a, b = a.to(F8), b.to(F8)
    one = lambda *s: torch.full(s, 127, dtype=torch.uint8, device="cuda").view(E8)  # noqa: E731
    z = torch.zeros(n, ld)
    z[:, :m] = negative(n, m, 2)
    c = torch.empty(n, ld, device="cuda")
    b2.b2_gemm_f8_act("T", "N", m, n, k, 0.25, a, k, one(-(-m // 128), -(-k // 128)), -(-k // 128), 128, b, k, one(n, -(-k // 128)), -(-k // 128), 1, b2.ACT_GELU | b2.ACT_GRADIENT, None, z.cuda(), ld,
                      None, ld, c, ld, None, m, None, 1)
    z = np64(z[:, :m])
    want = ffn.act_slope(z, "gelu")
    off = np.abs(np64(c[:, :m]) / 16 - want) / allowed(z, want)
    assert off.max() <= 1, (off.max(), z.flat[off.argmax()])
