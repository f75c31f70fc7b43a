"""The 8-bit result of a product with an epilogue over long k: it is the rounding of c, but for numbers next to a border of two e4m3 numbers.

Tolerance, derived before the first run: the tensor core adds 32 products at a time to a sum in fp32 and truncates, which takes less than 2^-23 of the sum each time; sums move to
fp32 registers every 4096 of k: 128 additions, 128 * 2^-23 = 1.53e-5 of a sum of terms of one sign; joining 16 such sums, the shares of a split and the product with alpha 32 roundings of
2^-24: 2e-6.  So a number that is further than 1.8e-5 of itself from a border has to be the definition's, where the block's scale is the definition's (or its largest magnitude within as much of one of
the rule's).  Sums over 65536 at once would be off by 6e-5."""
import pytest
import torch

pytestmark = pytest.mark.gpu
F8, E8 = torch.float8_e4m3fn, torch.float8_e8m0fnu
OFF = 1.8e-5


@pytest.mark.parametrize("gradient", [False, True])
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("m,n", [(20000, 8), (19072, 40), (384, 200), (1536, 1600), (1608, 1600), (1603, 1500)])
def test_long_sums(b2, m, n, dt, gradient):
    k = 65536
    g = torch.Generator(device="cuda").manual_seed(m)
    kb, mb = k // 128, -(-m // 128)
    a, b = (torch.randint(8, 120, (r, k), dtype=torch.uint8, device="cuda", generator=g).view(F8) for r in (m, n))  # positive, 2^-6 to 240
    sa, sb = (torch.randint(112, 114, (r, kb), dtype=torch.uint8, device="cuda", generator=g).view(E8) for r in (mb, n))
    z = torch.ones(n, m, dtype=dt, device="cuda")  # relu's derivative is 1
    q, s = torch.empty(n, m, dtype=F8, device="cuda"), torch.empty(n, mb, dtype=E8, device="cuda")
    b2.b2_gemm_f8_act("T", "N", m, n, k, 1.0, a, k, sa, kb, 128, b, k, sb, kb, 1, b2.ACT_RELU | (b2.ACT_GRADIENT if gradient else 0), None, z, m, None, m, None, m, q, m, s, mb)
    assert b2.b2_device_status() == 0
    want = torch.zeros(n, m, dtype=torch.float64, device="cuda")
    for k0 in range(0, k, 4096):
        at, blocks = slice(k0, k0 + 4096), slice(k0 // 128, k0 // 128 + 32)
        aa = a[:, at].double().view(m, 32, 128) * sa[:, blocks].float().double().repeat_interleave(128, 0)[:m, :, None]
        bb = b[:, at].double().view(n, 32, 128) * sb[:, blocks].float().double()[:, :, None]
        want += bb.view(n, -1) @ aa.view(m, -1).t()
    scale = s.float().double().repeat_interleave(128, 1)[:, :m]
    most = torch.nn.functional.pad(want, (0, mb * 128 - m)).view(n, mb, 128).amax(2)
    assert bool(((most * (1 + OFF) > 224 * s.float()) & (most * (1 - OFF) <= 448 * s.float())).all())
    y = want / scale  # positive and at most 448 (1 + OFF)
    step = torch.exp2(torch.floor(torch.log2(y.clamp(min=2.0**-6))) - 3)
    to = y / step
    clear = ((to - torch.floor(to) - 0.5).abs() * step > OFF * y) & (y < 448)  # from the border half way between two numbers
    right = torch.round(to) * step  # never half way
    off = (q.float().double() != right) & clear
    assert clear.float().mean() > 0.998 and int(off.sum()) == 0, int(off.sum())
