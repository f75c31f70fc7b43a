"""The 8-bit operators on the GPU against their definitions in 64 bits (oracle/f8.py).

Tolerances, u = 2^-24 (fp32), all derived before the first run:
- quantisation of given numbers is exact arithmetic (division by a power of two, one rounding): bit for bit.
- norm: the sum of squares of d terms in any order is within (d+1)u relative, rstd within half of that and three
  roundings, y with two more: |y - y_ref| <= ((d+1)/2 + 6) u |y_ref| =: e.  Then |q s - y_ref| <= e + half a step of e4m3
  at y (2^-4 |y|, or s 2^-10 below the normal range).  h is one fp32 addition and one rounding: bit for bit.
- backward: mean(g xh) is within (d+6)u of the mean of magnitudes; dx within 6u of its terms beside that, dw within (t+4)u of
  its sum of magnitudes; a result in bf16 adds 2^-8 of itself.
- products: the tensor core adds exact products of e4m3 (bf16 times e4m3-valued bf16) numbers in fp32 and may truncate
  (2u each), scales and their products and sums over blocks round 4 times per block: |C - C_ref| <= 2(k + 4 kb + 4) u S
  with S the sum of magnitudes, alpha and beta included; bf16 results 2^-8 |C_ref| more.  Integers times powers
  of two are exact as long as all sums fit 24 bits."""
import numpy as np
import pytest
import torch

from oracle import f8
from paper_1611_08035_b200 import binding as b2m

pytestmark = pytest.mark.gpu
U = 2.0**-24
BF, F32 = torch.bfloat16, torch.float32
F8, E8 = torch.float8_e4m3fn, torch.float8_e8m0fnu


def rand(shape, seed, dt=F32, spread=1.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(*shape, generator=g) * torch.exp(spread * torch.randn(shape[0], 1, generator=g))
    return x.to(dt)


def stored(x, ld, poison=float("nan"), offset=0):
    """x [cols][rows] on the GPU with columns of ld elements, `offset` elements into an allocation; poison everywhere else."""
    flat = torch.full((offset + x.shape[0] * ld,), poison, dtype=F32).to(x.dtype) if x.element_size() > 1 else \
        torch.full((offset + x.shape[0] * ld,), 0x7F, dtype=torch.uint8)
    flat[offset:].view(x.shape[0], ld)[:, : x.shape[1]] = x if x.element_size() > 1 else x.view(torch.uint8)
    return flat.cuda()[offset:].view(x.dtype)


def out_buffer(cols, ld, dt, offset=0):
    raw = torch.full(((offset + cols * ld) * dt.itemsize,), 0xA5, dtype=torch.uint8, device="cuda")
    return raw[offset * dt.itemsize :].view(dt)


def padding_untouched(buf, cols, rows, ld):
    b = buf.view(torch.uint8).view(cols, ld * buf.element_size())[:, rows * buf.element_size() :]
    return bool((b == 0xA5).all())


def q_values(q, d):
    return f8.E4M3[q.view(torch.uint8).view(-1, q.shape[-1] if q.dim() > 1 else d).cpu().numpy()]


def np64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def step_bound(y, s):
    return np.maximum(np.abs(y) * 2.0**-4, s * 2.0**-10)


# ---- quantisation -----------------------------------------------------------------------------------------------
QUANT = [(1, 1, 1, 0), (128, 1, 1, 0), (127, 3, 1, 0), (129, 5, 1, 0), (1003, 9, 1, 0), (1024, 33, 1, 8), (333, 17, 1, 3), (4104, 130, 1, 0),
         (1, 1, 128, 0), (128, 128, 128, 0), (127, 129, 128, 0), (300, 200, 128, 4), (257, 127, 128, 1)]


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("d,t,block,pad", QUANT)
def test_quant_bit_for_bit(b2, d, t, block, pad, dt):
    x = rand((t, d), d + t, dt, 3.0)
    if t > 2:
        x[1] = 0
    ld, nb, offset = d + pad, -(-d // 128), pad % 2
    q, s = out_buffer(t, ld, F8, offset), out_buffer(-(-t // block), nb + 1, E8)
    b2.b2_quant_f8(d, t, block, stored(x, ld, offset=offset), ld, q, ld, s, nb + 1)
    want_q, want_s = f8.quantise(np64(x), block)
    assert np.array_equal(q.view(torch.uint8).view(t, ld)[:, :d].cpu().numpy(), want_q)
    assert np.array_equal(s.view(torch.uint8).view(-1, nb + 1)[:, :nb].cpu().numpy(), want_s)
    assert padding_untouched(q, t, d, ld) and padding_untouched(s, -(-t // block), nb, nb + 1)


@pytest.mark.parametrize("block", [1, 128])
def test_quant_extremes(b2, block):
    """Zeros of both signs, subnormal and huge blocks, exact powers, NaN and infinities confined to their block."""
    d, t = 384, 6
    x = torch.zeros(t, d)
    x[0, :128], x[0, 5] = -0.0, 0.0
    x[1, :128] = 1e-41
    x[1, 130], x[1, 131] = 2.0**-120 * 1.5, 2.0**-126
    x[2, :128] = torch.finfo(F32).max
    x[2, 128:256] = 448.0
    x[3, :128], x[3, 7] = 1.0, float("nan")
    x[3, 128:256], x[3, 128] = 3.0, 448.0000305
    x[4, 200] = float("inf")
    x[5, 300] = float("-inf")
    q, s = out_buffer(t, d, F8), out_buffer(-(-t // block), 3, E8)
    b2.b2_quant_f8(d, t, block, x.cuda(), d, q, d, s, 3)
    want_q, want_s = f8.quantise(np64(x), block)
    assert np.array_equal(q.view(torch.uint8).view(t, d).cpu().numpy(), want_q)
    assert np.array_equal(s.view(torch.uint8).view(-1, 3).cpu().numpy(), want_s)


# ---- norm -------------------------------------------------------------------------------------------------------
NORM = [(1, 1, 0), (8, 3, 0), (127, 2, 0), (128, 5, 0), (250, 301, 0), (256, 9, 16), (512, 7, 0), (513, 303, 3), (1003, 1001, 24), (1024, 300, 0),
        (2048, 4, 0), (2056, 310, 8), (4096, 8, 0), (4096, 305, 0), (4100, 3, 1), (8192, 2, 0), (8192, 300, 0), (8200, 300, 0), (16384, 3, 0),
        (16390, 2, 2), (40003, 2, 0)]


@pytest.mark.parametrize("dt,res", [(BF, True), (BF, False), (F32, True)])
@pytest.mark.parametrize("d,t,pad", NORM)
def test_norm(b2, d, t, pad, dt, res):
    eps, ld, nb, offset = 1e-5, d + pad, -(-d // 128), pad % 2
    x, r = rand((t, d), d, dt), rand((t, d), t + 1, dt) if res else None
    w = (1 + 0.1 * rand((1, d), 5, spread=0.0)[0]).to(dt)
    q, s, h, rstd = out_buffer(t, ld, F8, offset), out_buffer(t, nb + 1, E8), out_buffer(t, ld, dt, offset) if res else None, out_buffer(t, 1, F32)
    b2.b2_rmsnorm_f8(d, t, stored(x, ld, offset=offset), ld, stored(r, ld, offset=offset) if res else None, ld, w.cuda(), eps, h, ld, q, ld, s, nb + 1, rstd)
    _, want_rstd, y = f8.rmsnorm(np64(x), np64(r) if res else None, np64(w), eps)
    rel = ((d + 1) / 2 + 6) * U
    assert np.all(np.abs(np64(rstd) - want_rstd) <= rel * want_rstd)
    if res:
        assert torch.equal(h.view(t, ld)[:, :d].cpu(), (x.float() + r.float()).to(dt)) and padding_untouched(h, t, d, ld)
    sv = f8.e8m0(s.view(torch.uint8).view(t, nb + 1)[:, :nb].cpu().numpy())
    amax = np.stack([np.abs(y[:, 128 * j : 128 * j + 128]).max(1) for j in range(nb)], 1)
    assert np.all(amax * (1 - rel) <= 448 * sv) and np.all(amax * (1 + rel) > 224 * sv)
    got = f8.E4M3[q.view(torch.uint8).view(t, ld)[:, :d].cpu().numpy()] * f8.spread(sv, (t, d))
    e = rel * np.abs(y)
    assert np.all(np.abs(got - y) <= e + step_bound(np.abs(y) + e, f8.spread(sv, (t, d))))
    assert padding_untouched(q, t, d, ld) and padding_untouched(s, t, nb, nb + 1)


@pytest.mark.parametrize("which", ["x", "r"])
@pytest.mark.parametrize("d,t", [(256, 5), (4096, 3), (40000, 2)])
def test_norm_in_place(b2, d, t, which):
    x, r, w = rand((t, d), 1, BF).cuda(), rand((t, d), 2, BF).cuda(), torch.ones(d, dtype=BF, device="cuda")
    nb = -(-d // 128)
    outs = []
    for place in (False, True):
        xx, rr = x.clone(), r.clone()
        h = (xx if which == "x" else rr) if place else torch.empty_like(x)
        q, s = torch.empty(t, d, dtype=F8, device="cuda"), torch.empty(t, nb, dtype=E8, device="cuda")
        b2.b2_rmsnorm_f8(d, t, xx, d, rr, d, w, 1e-6, h, d, q, d, s, nb, None)
        outs.append((h.clone(), q.view(torch.uint8), s.view(torch.uint8)))
    assert all(torch.equal(a, b) for a, b in zip(*outs))


def test_norm_zeros_and_non_finite(b2):
    """A token of zeros gives zeros; one with a NaN or an infinity is NaN where the formula has NaN, and only there."""
    d, t = 384, 4
    x = rand((t, d), 3, F32)
    x[0] = 0
    x[1, 200] = float("nan")
    x[2, 200] = float("inf")
    q, s, rstd = torch.empty(t, d, dtype=F8, device="cuda"), torch.empty(t, 3, dtype=E8, device="cuda"), torch.empty(t, device="cuda")
    b2.b2_rmsnorm_f8(d, t, x.cuda(), d, None, 1, torch.ones(d, device="cuda"), 1e-5, None, 1, q, d, s, 3, rstd)
    qb, sb = q.view(torch.uint8).cpu(), s.view(torch.uint8).cpu()
    assert bool((qb[0] == 0).all()) and sb[0].tolist() == [127] * 3 and abs(rstd[0].item() * 1e-5**0.5 - 1) < 1e-6
    assert bool((qb[1] == 0x7F).all()) and sb[1].tolist() == [255] * 3
    # rstd is 0: finite features become 0, the infinite one 0 * inf = NaN, which takes its block
    assert sb[2].tolist() == [127, 255, 127] and bool((qb[2, 128:256] == 0x7F).all()) and bool(((qb[2, :128] & 0x7F) == 0).all())
    assert sb[3].max() < 255 and rstd[2].item() == 0


BWD = [(1, 1, 0), (8, 3, 0), (127, 5, 0), (128, 64, 0), (1003, 1001, 24), (1024, 300, 0), (2048, 17, 8), (2050, 40, 1), (4096, 33, 0), (8192, 600, 0),
       (8200, 5, 0), (16384, 9, 0), (16392, 3, 0), (20001, 6, 3)]


@pytest.mark.parametrize("dt,res", [(BF, True), (F32, False)])
@pytest.mark.parametrize("d,t,pad", BWD)
def test_norm_backward(b2, d, t, pad, dt, res):
    ld, offset = d + pad, pad % 2
    h, dy, dh = rand((t, d), d, dt), rand((t, d), 7, dt, 0.3), rand((t, d), 8, dt, 0.3) if res else None
    w = (1 + 0.1 * rand((1, d), 5, spread=0.0)[0]).to(dt)
    rstd = torch.rsqrt(h.float().square().mean(1) + 1e-5)
    dx, dw = out_buffer(t, ld, dt, offset), torch.full((d,), float("nan"), device="cuda")
    ws = torch.empty(b2.b2_rmsnorm_backward_workspace_bytes(d, t), dtype=torch.uint8, device="cuda")
    args = (d, t, stored(dy, ld, offset=offset), ld, stored(h, ld, offset=offset), ld, rstd.cuda(), w.cuda(),
            stored(dh, ld, offset=offset) if res else None, ld, dx, ld, dw, ws)
    b2.b2_rmsnorm_backward(*args)
    a = [np64(v) for v in (dy, h, rstd, w)]
    want_dx, want_dw = f8.rmsnorm_backward(*a, np64(dh) if res else None)
    g, xh, r = np.abs(a[0] * a[3]), np.abs(a[1] * a[2][:, None]), a[2][:, None]
    terms = r * (6 * g + (d + 12) * xh * np.mean(g * xh, 1, keepdims=True)) + (np.abs(np64(dh)) * 2 if res else 0)
    tol = U * terms + (2.0**-8 * np.abs(want_dx) if dt == BF else 0)
    got = np64(dx.view(t, ld)[:, :d])
    assert np.all(np.abs(got - want_dx) <= tol) and padding_untouched(dx, t, d, ld)
    assert np.all(np.abs(np64(dw) - want_dw) <= (t + 4) * U * np.sum(np.abs(a[0]) * xh, 0))
    # the same bits again, and with dx written over dy
    first = (dx.clone(), dw.clone())
    if dt == BF:
        over = args[2].clone()
        b2.b2_rmsnorm_backward(d, t, over, ld, *args[4:10], over, ld, dw, ws)
        assert torch.equal(over.view(t, ld)[:, :d], first[0].view(t, ld)[:, :d])
    else:
        b2.b2_rmsnorm_backward(*args)
        assert torch.equal(dx.view(torch.uint8), first[0].view(torch.uint8))
    assert torch.equal(dw, first[1])


def test_norm_backward_against_differences(b2):
    """dx and dw along random directions against central differences of the 64-bit norm."""
    t, d, eps = 37, 515, 1e-5
    x, w, dy = rand((t, d), 1, F32, 0.2), 1 + 0.1 * rand((1, d), 2, spread=0.0)[0], rand((t, d), 3, F32, 0.2)
    X, W, DY = np64(x), np64(w), np64(dy)
    rstd = torch.from_numpy(f8.rmsnorm(X, None, W, eps)[1]).float()
    dx, dw = torch.empty(t, d, device="cuda"), torch.empty(d, device="cuda")
    ws = torch.empty(b2.b2_rmsnorm_backward_workspace_bytes(d, t), dtype=torch.uint8, device="cuda")
    b2.b2_rmsnorm_backward(d, t, dy.cuda(), d, x.cuda(), d, rstd.cuda(), w.cuda(), None, d, dx, d, dw, ws)
    loss = lambda X, W: float(np.sum(DY * f8.rmsnorm(X, None, W, eps)[2]))  # noqa: E731
    rng = np.random.default_rng(0)
    for _ in range(5):
        vx, vw, st = rng.normal(size=(t, d)), rng.normal(size=d), 1e-5
        num_x, num_w = (loss(X + st * vx, W) - loss(X - st * vx, W)) / (2 * st), (loss(X, W + st * vw) - loss(X, W - st * vw)) / (2 * st)
        # rounding of the differences: 1e-16 * loss / step, of the gradients: 1e-5 of their magnitudes
        assert abs(num_x - np.sum(np64(dx) * vx)) <= 1e-5 * np.sum(np.abs(np64(dx) * vx))
        assert abs(num_w - np.sum(np64(dw) * vw)) <= 1e-5 * np.sum(np.abs(np64(dw) * vw))


def test_norm_backward_of_no_tokens(b2):
    dw = torch.full((130,), 7.0, device="cuda")
    e = torch.empty(0, 130, device="cuda")
    b2.b2_rmsnorm_backward(130, 0, e, 130, e, 130, torch.empty(0, device="cuda"), dw.clone(), None, 130, e, 130, dw, None)
    assert bool((dw == 0).all())


# ---- products -----------------------------------------------------------------------------------------------------
def operand(rows, k, contiguous_k, block, scale, seed, pad, offset, integers, exponents=(-6, 5)):
    """Values [rows][k], scales [.][kb] as numpy, and the stored tensors (operand, ld, scales, ld of the scales)."""
    g = torch.Generator().manual_seed(seed)
    v = torch.randint(-4, 5, (rows, k), generator=g).float() if integers else torch.randn(rows, k, generator=g) * 60
    q = v.to(F8)
    shape = (-(-rows // block), -(-k // 128))
    s = torch.exp2(torch.randint(*exponents, shape, generator=g).float())
    if scale == "f32" and not integers:
        s = s * (1 + torch.rand(shape, generator=g))
    vals, scales = np64(q.float()), np64(s)
    if not contiguous_k:
        q, s = q.view(torch.uint8).t().contiguous().view(F8), s.t().contiguous()
    s_ld = s.shape[1] + 1
    s_st = stored(s if scale == "f32" else s.to(E8).view(torch.uint8), s_ld)
    ld = q.shape[1] + pad
    return vals, scales, stored(q, ld, offset=offset), ld, s_st if scale == "f32" else s_st.view(torch.uint8).view(E8), s_ld


def run_gemm(b2, ta, tb, m, n, k, ba=128, bb=1, scale=("e8m0", "e8m0"), out=BF, alpha=1.0, beta=0.0, pad=(0, 0, 0), offset=(0, 0), integers=False, exponents=(-6, 5), exact=False,
             seed=0):
    A, sa, a_st, lda, sa_st, ldsa = operand(m, k, ta == "T", ba, scale[0], seed + 1, pad[0], offset[0], integers, exponents)
    B, sb, b_st, ldb, sb_st, ldsb = operand(n, k, tb == "N", bb, scale[1], seed + 2, pad[1], offset[1], integers, exponents)
    ldc = m + pad[2]
    C = out_buffer(n, ldc, out)
    old = None
    if beta != 0:
        old = (torch.randint(-4, 5, (n, m)).float() if integers else 1e4 * torch.randn(n, m, generator=torch.Generator().manual_seed(9))).to(out)
        C.view(n, ldc)[:, :m] = old.cuda()
    nws = b2.b2_gemm_f8_workspace_bytes(ta, tb, m, n, k, a_st, lda, b_st, ldb)
    ws = torch.empty(nws, dtype=torch.uint8, device="cuda") if nws else None
    b2.b2_gemm_f8(ta, tb, m, n, k, alpha, a_st, lda, sa_st, ldsa, ba, b_st, ldb, sb_st, ldsb, bb, beta, C, ldc, ws)
    assert b2.b2_device_status() == 0
    want, S = f8.gemm(A, sa, ba, B, sb, bb)
    check_product(C, want, S, m, n, k, -(-k // 128), ldc, out, alpha, beta, old, exact)


def check_product(C, want, S, m, n, k, kb, ldc, out, alpha, beta, old, exact):
    want, S = alpha * want, abs(alpha) * S
    if beta != 0:
        want, S = want + beta * np64(old), S + abs(beta) * np.abs(np64(old))
    got = np64(C.view(n, ldc)[:, :m])
    if exact and out == F32:
        assert np.array_equal(got, want)
    else:
        tol = 2 * (k + 4 * kb + 4) * U * S + (2.0**-8 * np.abs(want) if out == BF else 0)
        assert np.all(np.abs(got - want) <= tol)
    assert padding_untouched(C, n, m, ldc)


GEMM = [("T", "N", 1, 1, 1), ("T", "N", 128, 1, 128), ("T", "N", 129, 3, 127), ("T", "N", 1000, 16, 260), ("T", "N", 257, 17, 1031), ("T", "N", 640, 33, 4096),
        ("T", "N", 300, 64, 513), ("T", "N", 130, 65, 128), ("T", "N", 1001, 999, 1003), ("T", "N", 384, 256, 3000), ("T", "N", 2300, 2100, 300),
        ("N", "N", 1, 2, 3), ("N", "N", 1001, 999, 1003), ("N", "N", 129, 5, 130), ("N", "N", 2304, 2176, 272),
        ("T", "T", 70, 20, 140), ("T", "T", 1001, 300, 257), ("N", "T", 200, 400, 600), ("N", "T", 33, 1, 65), ("T", "T", 2304, 2176, 130)]


@pytest.mark.parametrize("out,alpha,beta", [(BF, 1.0, 0.0), (F32, 1.5, -0.5)])
@pytest.mark.parametrize("ta,tb,m,n,k", GEMM)
def test_gemm(b2, ta, tb, m, n, k, out, alpha, beta):
    run_gemm(b2, ta, tb, m, n, k, out=out, alpha=alpha, beta=beta, pad=(0, 0, 3), seed=m + n)


@pytest.mark.parametrize("scale", [("e8m0", "e8m0"), ("f32", "f32"), ("f32", "e8m0"), ("e8m0", "f32")])
@pytest.mark.parametrize("ba,bb", [(128, 1), (1, 1), (1, 128), (128, 128)])
@pytest.mark.parametrize("ta,tb,m,n,k", [("T", "N", 300, 20, 400), ("T", "N", 300, 200, 400), ("N", "T", 272, 200, 400), ("T", "N", 4700, 1100, 400)])
def test_gemm_scales(b2, ta, tb, m, n, k, ba, bb, scale):
    run_gemm(b2, ta, tb, m, n, k, ba, bb, scale, out=F32, pad=(16, 16, 1), seed=3)


INTEGERS = [("T", "N", 200, 9, 1003), ("N", "N", 333, 130, 500), ("T", "N", 2304, 2176, 500), ("T", "T", 200, 50, 700)]


@pytest.mark.parametrize("scale", ["e8m0", "f32"])
@pytest.mark.parametrize("ta,tb,m,n,k", INTEGERS)
def test_gemm_integers_are_exact(b2, ta, tb, m, n, k, scale):
    """Scales of 1/2, 1 and 2: every term is a multiple of 1/4 and every sum below 2^18, 20 of fp32's 24 bits."""
    run_gemm(b2, ta, tb, m, n, k, scale=(scale, scale), out=F32, alpha=2.0, beta=1.0, integers=True, exponents=(-1, 2), exact=True, pad=(8, 40, 0))


@pytest.mark.parametrize("scale", ["e8m0", "f32"])
@pytest.mark.parametrize("ta,tb,m,n,k", INTEGERS)
def test_gemm_integers_wide_scales(b2, ta, tb, m, n, k, scale):
    """Scales from 2^-6 to 2^4: sums of multiples of 2^-12 up to 2^22, more bits than fp32 has, so within the bound only."""
    run_gemm(b2, ta, tb, m, n, k, scale=(scale, scale), out=F32, alpha=2.0, beta=1.0, integers=True, pad=(8, 40, 0))


@pytest.mark.parametrize("pad,offset", [((1, 0, 0), (0, 0)), ((0, 3, 0), (0, 0)), ((0, 0, 0), (5, 0)), ((7, 9, 1), (1, 15))])
@pytest.mark.parametrize("ta,tb", [("T", "N"), ("N", "T")])
def test_gemm_unaligned(b2, ta, tb, pad, offset):
    run_gemm(b2, ta, tb, 160, 144, 320, pad=pad, offset=offset)


def test_gemm_quick_returns(b2):
    q, s = torch.zeros(4, 128, dtype=torch.uint8, device="cuda").view(F8), torch.full((4, 1), 255, dtype=torch.uint8, device="cuda").view(E8)
    for dt in (F32, BF):
        C = torch.full((4, 4), float("nan"), dtype=dt, device="cuda")
        b2.b2_gemm_f8("T", "N", 4, 4, 0, 1.0, q, 128, s, 1, 1, q, 128, s, 1, 1, 0.0, C, 4)  # k == 0, beta == 0: zeros, C not read
        assert bool((C == 0).all())
        C.fill_(3.0)
        b2.b2_gemm_f8("T", "N", 4, 4, 128, 0.0, q, 128, s, 1, 1, q, 128, s, 1, 1, 0.5, C, 4)  # alpha == 0: operands not read
        assert bool((C == 1.5).all())
        b2.b2_gemm_f8("T", "N", 4, 4, 128, 0.0, q, 128, s, 1, 1, q, 128, s, 1, 1, 1.0, C, 4)
        b2.b2_gemm_f8("T", "N", 0, 4, 128, 1.0, q, 128, s, 1, 1, q, 128, s, 1, 1, 0.0, C, 4)
        assert bool((C == 1.5).all())


@pytest.mark.parametrize("scale", ["e8m0", "f32"])
@pytest.mark.parametrize("n", [5, 300])
def test_gemm_non_finite(b2, n, scale):
    """A NaN number or a NaN scale reaches exactly the rows and columns of C that it enters; nothing else does."""
    m, k = 260, 300
    g = torch.Generator().manual_seed(0)
    a, b = torch.randint(0, 0x70, (m, k + 4), generator=g, dtype=torch.uint8), torch.randint(0, 0x70, (n, k + 4), generator=g, dtype=torch.uint8)
    a[7, 299], b[2, 0] = 0x7F, 0xFF
    sa, sb = torch.full((3, 3), 127, dtype=torch.uint8), torch.full((n, 3), 127, dtype=torch.uint8)
    sb[4, 1], sa[2, 2] = 255, 255
    to = lambda s: s.cuda().view(E8) if scale == "e8m0" else torch.where(s == 255, float("nan"), 1.0).cuda()  # noqa: E731
    C = torch.empty(n, m, device="cuda")
    ws = torch.empty(b2.b2_gemm_f8_workspace_bytes("T", "N", m, n, k, a, k + 4, b, k + 4) or 1, dtype=torch.uint8, device="cuda")
    b2.b2_gemm_f8("T", "N", m, n, k, 1.0, a.cuda().view(F8), k + 4, to(sa), 3, 128, b.cuda().view(F8), k + 4, to(sb), 3, 1, 0.0, C, m, ws)
    want = torch.zeros(n, m, dtype=torch.bool)
    want[:, 7], want[2], want[4], want[:, 256:] = True, True, True, True
    assert torch.equal(torch.isnan(C).cpu(), want) and b2.b2_device_status() == 0


# ---- weight gradient ----------------------------------------------------------------------------------------------
def run_wgrad(b2, m, n, k, out=F32, alpha=1.0, beta=0.0, pad=(0, 0, 0), offset=(0, 0), integers=False, seed=0):
    g = torch.Generator().manual_seed(seed)
    q = (torch.randint(-4, 5, (k, m), generator=g).float() if integers else torch.randn(k, m, generator=g) * 60).to(F8)
    sb = torch.randint(121, 134, (k, -(-m // 128)), generator=g, dtype=torch.uint8)
    y = (torch.randint(-4, 5, (k, n), generator=g).float() if integers else torch.randn(k, n, generator=g)).to(BF)
    ldq, ldy, ldc, lds = m + pad[0], n + pad[1], m + pad[2], sb.shape[1] + 1
    q_st, y_st, s_st = stored(q, ldq, offset=offset[0]), stored(y, ldy, offset=offset[1]), stored(sb, lds).view(E8)
    C = out_buffer(n, ldc, out)
    old = None
    if beta != 0:
        old = torch.randint(-4, 5, (n, m)).to(out)
        C.view(n, ldc)[:, :m] = old.cuda()
    nws = b2.b2_wgrad_f8_workspace_bytes(m, n, k, q_st, ldq, y_st, ldy)
    ws = torch.empty(nws, dtype=torch.uint8, device="cuda") if nws else None
    b2.b2_wgrad_f8(m, n, k, alpha, q_st, ldq, s_st, lds, y_st, ldy, beta, C, ldc, ws)
    assert b2.b2_device_status() == 0
    want, S = f8.wgrad(np64(q.float()), f8.e8m0(sb.numpy()), np64(y))
    check_product(C, want, S, m, n, k, -(-k // 64), ldc, out, alpha, beta, old, integers)


WGRAD = [(1, 1, 1), (128, 128, 64), (129, 127, 65), (1003, 1001, 999), (16, 300, 5), (700, 24, 2050), (256, 128, 4200), (2304, 2200, 130), (2400, 4500, 63)]


@pytest.mark.parametrize("out,alpha,beta", [(F32, 1.0, 0.0), (BF, 0.5, 2.0), (F32, 1.0, 1.0)])
@pytest.mark.parametrize("m,n,k", WGRAD)
def test_wgrad(b2, m, n, k, out, alpha, beta):
    run_wgrad(b2, m, n, k, out, alpha, beta, pad=(0, 0, 3), seed=m)


@pytest.mark.parametrize("m,n,k", [(200, 136, 1003), (1003, 1001, 70), (2400, 4500, 100)])
def test_wgrad_integers_are_exact(b2, m, n, k):
    run_wgrad(b2, m, n, k, alpha=2.0, beta=1.0, integers=True, pad=(8, 8, 1))


@pytest.mark.parametrize("pad,offset", [((1, 0, 0), (0, 0)), ((0, 3, 0), (0, 0)), ((0, 0, 0), (3, 1)), ((16, 24, 2), (16, 8))])
def test_wgrad_strides(b2, pad, offset):
    run_wgrad(b2, 160, 136, 200, pad=pad, offset=offset)


def test_wgrad_every_number_and_scale(b2):
    """All 256 bytes of e4m3 under small, ordinary and large scales reach the product as they are (y = 1, one token)."""
    k, m = 1, 256
    bytes_ = torch.arange(256, dtype=torch.uint8).view(1, 256).cuda()
    y = torch.ones(1, 8, dtype=BF, device="cuda")
    for s in (3, 40, 127, 134, 135, 200, 239):
        C = torch.empty(8, m, device="cuda")
        sc = torch.full((1, 2), s, dtype=torch.uint8, device="cuda")
        b2.b2_wgrad_f8(m, 8, k, 1.0, bytes_.view(F8), 256, sc.view(E8), 2, y, 8, 0.0, C, m)
        want = f8.E4M3 * f8.e8m0(s)
        for j in (0, 7):
            assert np.array_equal(np64(C[j]), want, equal_nan=True), s
    sc = torch.tensor([[255, 127]], dtype=torch.uint8, device="cuda")
    b2.b2_wgrad_f8(m, 8, k, 1.0, torch.zeros_like(bytes_).view(F8), 256, sc.view(E8), 2, y, 8, 0.0, C, m)
    assert bool(torch.isnan(C[:, :128]).all()) and bool((C[:, 128:] == 0).all())


# ---- all of them ----------------------------------------------------------------------------------------------------
def test_other_stream_and_long_columns(b2):
    """Work goes to the current stream; columns far apart have offsets beyond 32 bits."""
    d, t, ld = 136, 1100, 4_000_016  # 4.4e9 elements
    x = torch.empty(t * ld, dtype=torch.uint8, device="cuda")  # numbers are spread over the whole allocation
    src = rand((t, d), 1, BF, 1.0)
    dense, small = src.cuda(), torch.empty(t, d, dtype=F8, device="cuda")
    s, s2 = torch.empty(t, 2, dtype=E8, device="cuda"), torch.empty(t, 2, dtype=E8, device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        b2.b2_quant_f8(d, t, 1, dense, d, x.view(F8), ld, s, 2)
        b2.b2_quant_f8(d, t, 1, dense, d, small, d, s2, 2)
        C1, C2 = torch.empty(8, t, device="cuda"), torch.empty(8, t, device="cuda")
        ws = torch.empty(b2.b2_gemm_f8_workspace_bytes("T", "N", t, 8, d, small, d, small, d) or 256, dtype=torch.uint8, device="cuda")
        b2.b2_gemm_f8("T", "N", t, 8, d, 1.0, x.view(F8), ld, s, 2, 1, small, d, s2, 2, 1, 0.0, C1, t, ws)
        b2.b2_gemm_f8("T", "N", t, 8, d, 1.0, small, d, s2, 2, 1, small, d, s2, 2, 1, 0.0, C2, t, ws)
    stream.synchronize()
    assert torch.equal(x.view(t, ld)[:, :d], small.view(torch.uint8)) and torch.equal(s.view(torch.uint8), s2.view(torch.uint8))
    assert torch.equal(C1, C2) and b2.b2_device_status() == 0


def test_call_forms(b2):
    """Positional, keyword and unchecked calls, refused types and refused arguments, whichever way the binding takes."""
    x = torch.randn(4, 128, device="cuda")
    q, s = torch.empty(4, 128, dtype=F8, device="cuda"), torch.empty(4, 1, dtype=E8, device="cuda")
    assert b2.b2_quant_f8(128, 4, 1, x, 128, q, 128, s, 1) == 0
    first = q.clone()
    assert b2.b2_quant_f8(128, 4, 1, x, 128, q, 128, s=s, lds=1) == 0 and torch.equal(q.view(torch.uint8), first.view(torch.uint8))
    for call in (lambda **kw: b2.b2_quant_f8(128, 4, 3, x, 128, q, 128, s, 1, **kw), lambda **kw: b2.b2_quant_f8(d=128, t=4, block=3, x=x, ldx=128, q=q, ldq=128, s=s, lds=1, **kw)):
        with pytest.raises(b2.B2Error) as e:
            call()
        assert e.value.status == -3
        assert call(check=False) == -3
    with pytest.raises(TypeError):
        b2.b2_quant_f8(128, 4, 1, x.half(), 128, q, 128, s, 1)
    with pytest.raises(TypeError):
        b2.b2_quant_f8(128, 4, 1, x.cpu(), 128, q, 128, s, 1)
    with pytest.raises(TypeError):
        b2.b2_quant_f8(128, 4, 1)
    C = torch.empty(4, 4, device="cuda")
    with pytest.raises(b2.B2Error) as e:  # an operand that needs a workspace, without one
        b2.b2_gemm_f8("T", "N", 4, 4, 100, 1.0, q, 100, s, 1, 1, q, 128, s, 1, 1, 0.0, C, 4)
    assert e.value.status == 1003
    with pytest.raises(TypeError):
        b2.b2_wgrad_f8(128, 4, 4, 1.0, q, 128, s, 1, x, 128, 0.0, C, 128)


WIDTHS = [264, 520, 776, 1100, 1152, 1536, 2080, 2560, 2561, 3184, 5120, 6272, 7176, 9000, 10240]


@pytest.mark.parametrize("dt,res", [(BF, True), (F32, False)])
@pytest.mark.parametrize("d", WIDTHS)
def test_norm_of_every_width(b2, d, dt, res):
    """More tokens than one for each CTA, by every number of warps that a token can take."""
    test_norm(b2, d, 320, 0, dt, res)
    test_norm_backward(b2, d, 2 * 1024 * 1024 // d + 400, 0, dt, res)


@pytest.mark.parametrize("d,t", [(520, 1700), (896, 2300), (1001, 2300)])
def test_norm_backward_of_many_short_tokens(b2, d, t):
    test_norm_backward(b2, d, t, 0, BF, True)
    test_norm_backward(b2, d, t, 0, F32, False)


@pytest.mark.parametrize("scale", ["e8m0", "f32"])
@pytest.mark.parametrize("out", [BF, F32])
@pytest.mark.parametrize("m,pad", [(2304, 0), (2302, 2), (2301, 3), (2303, 0)])
def test_gemm_adds_to_large_results(b2, m, pad, out, scale):
    """Tiles on pairs of CTAs added to C in whole 16-byte pieces, in parts of one, and one by one."""
    run_gemm(b2, "T", "N", m, 2176, 300, scale=(scale, scale), out=out, alpha=1.5, beta=-0.5, pad=(0, 0, pad), seed=4)


@pytest.mark.parametrize("m,n", [(200, 300), (300, 20), (2304, 2176)])
@pytest.mark.parametrize("k", [384, 500, 890, 1400])
def test_gemm_scales_in_words_and_bytes(b2, m, n, k):
    run_gemm(b2, "T", "N", m, n, k, seed=5)
    run_gemm(b2, "T", "N", m, n, k, ba=1, seed=6)


@pytest.mark.parametrize("k", [1, 2, 3, 15, 17, 19, 20, 31, 33, 47])
def test_gemm_of_short_odd_columns(b2, k):
    run_gemm(b2, "T", "N", 40, 70, k, pad=(0, 1, 0), offset=(3, 0), out=F32, integers=True, exponents=(-1, 2), exact=True)
    run_gemm(b2, "N", "T", k, k + 1, 140, pad=(1, 0, 0), offset=(0, 7), out=F32, integers=True, exponents=(-1, 2), exact=True)


@pytest.mark.parametrize("out,beta", [(BF, 2.0), (F32, 0.0), (F32, 1.0)])
@pytest.mark.parametrize("m,n,k", [(2304, 1536, 200), (2301, 1533, 130), (384, 1536, 1344), (288, 648, 6512), (640, 640, 2048)])
def test_wgrad_of_every_split(b2, m, n, k, out, beta):
    test_wgrad(b2, m, n, k, out, 0.5, beta)
