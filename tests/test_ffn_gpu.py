"""The products with an epilogue and the activation's backward pass on the GPU against their definitions in 64 bits (oracle/f8.py, oracle/ffn.py).

Tolerances, u = 2^-24, derived before the first run:
- the product's sum v: 2 (k + 4 kb + 4) u S =: e, S the sum of magnitudes with alpha (as for the product alone);
- z = v + bias: e + u |z|;
- act(z): no slope exceeds 1.13; the function itself is within 2^-20 max(1, |value|) (stated in the header);
- gradient form: |v| 2^-18 + e |slope|, slopes within 2^-18, with the product's rounding u |c|;
- plus the residual: u |c|;
- storing: half a step, u for fp32, 2^-8 for bf16, relative; e4m3: 2^-4, or s 2^-10 below its normal range.
Integer sums with scales of 1 and no function are exact.  db: t numbers, each with its own error, added in any order: (t + 4) u times the sum of magnitudes."""
import numpy as np
import pytest
import torch

from oracle import f8, ffn

pytestmark = pytest.mark.gpu
U = 2.0**-24
BF, F32 = torch.bfloat16, torch.float32
F8, E8 = torch.float8_e4m3fn, torch.float8_e8m0fnu
HALF = {BF: 2.0**-8, F32: U}


def stored(x, ld, offset=0):
    """x [cols][rows] on the GPU with columns of ld elements, `offset` elements into an allocation; NaN everywhere else."""
    one = x.element_size() == 1
    flat = torch.full((offset + x.shape[0] * ld,), 0x7F, dtype=torch.uint8) if one else torch.full((offset + x.shape[0] * ld,), float("nan"), dtype=x.dtype)
    flat[offset:].view(x.shape[0], ld)[:, : x.shape[1]] = x.view(torch.uint8) if one else x
    return flat.cuda()[offset:].view(x.dtype)


def buffer(cols, ld, dt, offset=0):
    raw = torch.full(((offset + cols * ld) * dt.itemsize,), 0xA5, dtype=torch.uint8, device="cuda")
    return raw[offset * dt.itemsize :].view(dt)


def rows_of(buf, cols, rows, ld):
    """The matrix in a buffer, whose padding has to be what it was."""
    b = buf.view(torch.uint8).view(cols, ld * buf.element_size())
    assert bool((b[:, rows * buf.element_size() :] == 0xA5).all()), "padding was written"
    return buf.view(torch.uint8).view(cols, -1)[:, : rows * buf.element_size()].contiguous().view(buf.dtype).view(cols, rows)


def np64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def check_quantised(q, s, want, e):
    """e4m3 numbers and scales of a result that is within e of `want`."""
    t, d = want.shape
    sv = f8.e8m0(s.view(torch.uint8).cpu().numpy())
    nb = sv.shape[1]
    amax = np.stack([np.abs(want[:, 128 * j : 128 * j + 128]).max(1) for j in range(nb)], 1)
    em = np.stack([e[:, 128 * j : 128 * j + 128].max(1) for j in range(nb)], 1)
    assert np.all(np.maximum(amax - em, 0) <= 448 * sv) and np.all((amax + em > 224 * sv) | (sv == 1.0))
    got = f8.E4M3[q.view(torch.uint8).cpu().numpy()] * f8.spread(sv, (t, d))
    step = np.maximum((np.abs(want) + e) * 2.0**-4, f8.spread(sv, (t, d)) * 2.0**-10)
    assert np.all(np.abs(got - want) <= e + step)


def run_product(b2, m, n, k, act="gelu", gradient=False, ta="T", tb="N", scale="e8m0", ba=128, bb=1, out=BF, alpha=1.0, bias=True, z=True, res=True, c=True, q=True, pad=0, offset=0,
                seed=0, integers=False):
    g = torch.Generator().manual_seed(seed + m + n)
    kb, mb = -(-k // 128), -(-m // 128)
    a = (torch.randint(-3, 4, (m, k), generator=g).float() if integers else torch.randn(m, k, generator=g) * 4).to(F8)
    b = (torch.randint(-3, 4, (n, k), generator=g).float() if integers else torch.randn(n, k, generator=g) * 4).to(F8)
    unit = 1.0 if integers else 0.25 * k**-0.5

    def scales(rows, block, low):
        if integers:
            return torch.full((-(-rows // block), kb), 127, dtype=torch.uint8).view(E8) if scale == "e8m0" else torch.ones(-(-rows // block), kb)
        if scale == "e8m0":
            return torch.randint(low, low + 3, (-(-rows // block), kb), generator=g, dtype=torch.uint8).view(E8)
        return 2.0 ** (low - 126) * (0.5 + torch.rand(-(-rows // block), kb, generator=g))

    sa, sb = scales(m, ba, 126), scales(n, bb, 125)
    transposed = lambda x: x.view(torch.uint8).t().contiguous().view(x.dtype) if x.element_size() == 1 else x.t().contiguous()  # noqa: E731
    A, SA = (a, sa) if ta == "T" else (transposed(a), transposed(sa))
    B, SB = (b, sb) if tb == "N" else (transposed(b), transposed(sb))
    alpha = alpha * unit
    ld = m + pad
    bias_ = torch.randn(m, generator=g) if bias and not gradient else None
    z_in = (torch.randn(n, m, generator=g) * 2).to(out) if gradient else None
    r_ = torch.randn(n, m, generator=g).to(out) if res else None
    if integers:
        bias_, r_ = (None if x is None else torch.round(x * 4) for x in (bias_, r_))
    Z = stored(z_in, ld, offset) if gradient else buffer(n, ld, out, offset) if z else None
    C, Q, S = buffer(n, ld, out, offset) if c else None, buffer(n, ld, F8, offset) if q else None, buffer(n, mb + 1, E8) if q else None
    code = getattr(b2, "ACT_" + act.upper()) | (b2.ACT_GRADIENT if gradient else 0)
    a_st, b_st = stored(A, A.shape[1] + pad, offset), stored(B, B.shape[1] + pad, offset)
    sa_st, sb_st = SA.cuda(), SB.cuda()
    nws = b2.b2_gemm_f8_workspace_bytes(ta, tb, m, n, k, a_st, A.shape[1] + pad, b_st, B.shape[1] + pad)
    ws = torch.empty(nws, dtype=torch.uint8, device="cuda") if nws else None
    b2.b2_gemm_f8_act(ta, tb, m, n, k, alpha, a_st, A.shape[1] + pad, sa_st, SA.shape[1], ba, b_st, B.shape[1] + pad, sb_st, SB.shape[1], bb, code,
                      None if bias_ is None else bias_.cuda(), Z, ld, None if r_ is None else stored(r_, ld, offset), ld, C, ld, Q, ld, S, mb + 1, ws)
    assert b2.b2_device_status() == 0
    alpha = float(np.float32(alpha))
    want, mags = f8.gemm(np64(a.float()), np64(sa.float()), ba, np64(b.float()), np64(sb.float()), bb)
    v, e = alpha * want, 2 * (k + 4 * kb + 4) * U * abs(alpha) * mags
    if gradient:
        slope = ffn.act_slope(np64(z_in), act)
        e = np.abs(v) * (2.0**-18 if act not in ("none", "relu") else 0) + e * np.abs(slope)
        v = v * slope
        e = e + U * np.abs(v)
    else:
        if bias_ is not None:
            v = v + np64(bias_)
            e = e + U * (np.abs(v) + e)
        if z:
            got = np64(rows_of(Z, n, m, ld))
            assert np.all(np.abs(got - v) <= e + HALF[out] * (np.abs(v) + e)) and (not integers or out is BF or np.array_equal(got, v))
        v = ffn.act(v, act)
        e = 1.13 * e + (0 if act in ("none", "relu") else 2.0**-20 * np.maximum(1, np.abs(v)))
    if r_ is not None:
        v = v + np64(r_)
        e = e + U * (np.abs(v) + e)
    if c:
        got = np64(rows_of(C, n, m, ld))
        assert np.all(np.abs(got - v) <= e + HALF[out] * (np.abs(v) + e)), np.max(np.abs(got - v) / (e + HALF[out] * (np.abs(v) + e)))
        assert not integers or out is BF or act != "none" or np.array_equal(got, v)
    if q:
        check_quantised(rows_of(Q, n, m, ld), rows_of(S, n, mb, mb + 1), v, e)


# single CTAs: decoding (rows are features) with every width, with and without a split; whole tiles, halves of a block, split and not; pairs of CTAs
SIZES = [(1, 1, 1), (130, 1, 300), (127, 8, 128), (300, 5, 2050), (1003, 17, 515), (260, 40, 1100), (20000, 8, 130), (19100, 33, 70), (256, 64, 4096),
         (128, 65, 128), (200, 130, 257), (333, 300, 1003), (512, 512, 2048), (1100, 900, 260), (1601, 1500, 300), (2304, 1800, 129), (513, 5000, 1100)]


@pytest.mark.parametrize("scale", ["e8m0", "f32"])
@pytest.mark.parametrize("out", [BF, F32])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_forward(b2, m, n, k, out, scale):
    run_product(b2, m, n, k, "gelu", out=out, scale=scale, pad=3 if m % 2 else 8)


@pytest.mark.parametrize("out", [BF, F32])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_gradient(b2, m, n, k, out):
    run_product(b2, m, n, k, "silu", gradient=True, ta="N", out=out, res=m % 3 == 0, pad=0 if m % 2 else 16)


@pytest.mark.parametrize("gradient", [False, True])
@pytest.mark.parametrize("act", ffn.ACTS)
@pytest.mark.parametrize("m,n,k", [(260, 7, 200), (300, 200, 130), (1600, 1500, 140)])
def test_functions(b2, m, n, k, act, gradient):
    run_product(b2, m, n, k, act, gradient=gradient, out=F32, scale="f32" if n == 200 else "e8m0", ba=1 if n == 200 else 128, alpha=1.5, seed=3)


@pytest.mark.parametrize("bias,z,res,c,q", [(False, False, False, True, False), (True, False, False, True, False), (False, True, False, True, False), (False, False, True, True, False),
                                            (False, False, False, False, True), (True, True, False, False, True), (False, False, True, True, True), (True, True, True, True, False)])
@pytest.mark.parametrize("m,n,k", [(260, 7, 200), (500, 64, 3000), (300, 200, 130), (520, 500, 2100), (1600, 1500, 140)])
def test_parts(b2, m, n, k, bias, z, res, c, q):
    run_product(b2, m, n, k, "gelu_tanh", bias=bias, z=z, res=res, c=c, q=q, seed=5)


@pytest.mark.parametrize("pad,offset", [(1, 0), (5, 3), (0, 1), (16, 16), (8, 8)])
@pytest.mark.parametrize("m,n,k", [(260, 7, 200), (500, 20, 3000), (300, 200, 130), (520, 500, 2100), (512, 512, 512), (1600, 1500, 140)])
def test_strides(b2, m, n, k, pad, offset):
    run_product(b2, m, n, k, "silu", pad=pad, offset=offset, out=BF if pad != 5 else F32, seed=7)


@pytest.mark.parametrize("scale,out", [("e8m0", BF), ("e8m0", F32), ("f32", BF)])
@pytest.mark.parametrize("m", [1601, 1602, 1604, 1606, 1607, 1608, 1609, 1612, 1616])
def test_padding_behind_odd_sizes(b2, m, scale, out):
    """Aligned columns whose last number is within 16 bytes: what lies between there and the next column stays as it is, in every result."""
    for parts in ({"q": True, "z": True}, {"q": False, "z": False}, {"q": False, "gradient": True, "ta": "N"}):
        run_product(b2, m, 1500, 140, "silu", scale=scale, out=out, pad=(-m) % 16 + 16, seed=11, **parts)


@pytest.mark.parametrize("ta,tb,ba,bb", [("T", "T", 1, 128), ("N", "T", 128, 1), ("N", "N", 1, 1), ("T", "N", 128, 128)])
@pytest.mark.parametrize("m,n,k", [(260, 7, 200), (300, 200, 130), (1600, 1500, 140)])
def test_layouts(b2, m, n, k, ta, tb, ba, bb):
    run_product(b2, m, n, k, "relu", ta=ta, tb=tb, ba=ba, bb=bb, scale="f32" if ba == bb else "e8m0", seed=9)


@pytest.mark.parametrize("scale", ["e8m0", "f32"])
@pytest.mark.parametrize("m,n,k", [(260, 7, 200), (500, 20, 3000), (300, 200, 130), (520, 500, 2100), (1600, 1500, 140)])
def test_integers_are_exact(b2, m, n, k, scale):
    run_product(b2, m, n, k, "none", out=F32, scale=scale, integers=True, q=False, pad=1)


@pytest.mark.parametrize("out", [BF, F32])
@pytest.mark.parametrize("alpha,k", [(0.0, 130), (1.0, 0)])
def test_sums_of_nothing(b2, alpha, k, out):
    """alpha or k 0: the operands are not read; everything else goes on."""
    m, n = 300, 70
    nan = torch.full((m, 256), 0x7F, dtype=torch.uint8, device="cuda").view(F8)
    s = torch.full((m, 2), 255, dtype=torch.uint8, device="cuda").view(E8)
    bias, r = torch.randn(m), torch.randn(n, m).to(out)
    z, c, q, sq = buffer(n, m, out), buffer(n, m, out), buffer(n, m, F8), buffer(n, 3, E8)
    b2.b2_gemm_f8_act("T", "N", m, n, k, alpha, nan, 256, s, 2, 1, nan, 256, s, 2, 1, b2.ACT_GELU, bias.cuda(), z, m, r.cuda(), m, c, m, q, m, sq, 3)
    v = np.broadcast_to(np64(bias), (n, m))
    assert np.all(np.abs(np64(z.view(n, m)) - v) <= HALF[out] * np.abs(v))
    v = ffn.act(v, "gelu") + np64(r)
    e = 2.0**-20 * np.maximum(1, np.abs(v)) + U * np.abs(v)
    assert np.all(np.abs(np64(c.view(n, m)) - v) <= e + HALF[out] * (np.abs(v) + e))
    check_quantised(q.view(n, m), sq.view(n, 3), v, e)
    b2.b2_gemm_f8_act("T", "N", 0, n, 128, 1.0, nan, 256, s, 2, 1, nan, 256, s, 2, 1, 0, None, None, 1, None, 1, c, 1, None, 1, None, 1)
    b2.b2_gemm_f8_act("T", "N", m, 0, 128, 1.0, nan, 256, s, 2, 1, nan, 256, s, 2, 1, 0, None, None, m, None, m, c, m, None, 1, None, 1)
    assert np.all(np.abs(np64(c.view(n, m)) - v) <= e + HALF[out] * (np.abs(v) + e))


def plain_operands(m, n, k, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    a, b = torch.randn(m, k, device="cuda", generator=g).to(F8), torch.randn(n, k, device="cuda", generator=g).to(F8)
    kb = -(-k // 128)
    return a, torch.full((-(-m // 128), kb), 124, dtype=torch.uint8, device="cuda").view(E8), b, torch.full((n, kb), 124, dtype=torch.uint8, device="cuda").view(E8)


@pytest.mark.parametrize("out", [BF, F32])
@pytest.mark.parametrize("m,n,k", [(256, 7, 256), (512, 20, 4096), (304, 200, 128), (528, 500, 2176), (1600, 1504, 128), (301, 203, 128)])
def test_in_place(b2, m, n, k, out):
    """The residual in the place of the result, and in the gradient form the z that is read."""
    a, sa, b, sb = plain_operands(m, n, k)
    r = torch.randn(n, m, device="cuda").to(out)
    call = lambda act, z, r, c: b2.b2_gemm_f8_act("T", "N", m, n, k, 0.25, a, k, sa, sa.shape[1], 128, b, k, sb, sb.shape[1], 1, act, None, z, m, r, m, c, m, None, m, None, 1)  # noqa: E731
    apart, place = torch.empty_like(r), r.clone()
    call(b2.ACT_SILU, None, r, apart)
    call(b2.ACT_SILU, None, place, place)
    assert torch.equal(apart, place) and not torch.equal(place, r)
    z, dz = torch.randn(n, m, device="cuda").to(out), torch.empty_like(r)
    call(b2.ACT_GELU | b2.ACT_GRADIENT, z, r, dz)
    call(b2.ACT_GELU | b2.ACT_GRADIENT, z, r, z)
    assert torch.equal(z, dz)


@pytest.mark.parametrize("n", [5, 300, 1500])
def test_not_finite(b2, n):
    """A NaN in an operand reaches the rows and columns it enters; its blocks of 128 are NaN in 8 bits, the others are not.  Infinite and NaN residuals likewise."""
    m, k = 1700 if n == 1500 else 300, 256
    a, sa, b, sb = plain_operands(m, n, k)
    a.view(torch.uint8)[7, 200] = 0x7F
    r = torch.zeros(n, m, device="cuda")
    r[3, 140], r[1, 299] = float("inf"), float("nan")
    c, q, s = torch.empty(n, m, device="cuda"), torch.empty(n, m, dtype=F8, device="cuda"), torch.empty(n, -(-m // 128), dtype=E8, device="cuda")
    b2.b2_gemm_f8_act("T", "N", m, n, k, 0.25, a, k, sa, 2, 128, b, k, sb, 2, 1, b2.ACT_GELU, None, None, m, r, m, c, m, q, m, s, s.shape[1])
    bad = torch.zeros(n, m, dtype=torch.bool, device="cuda")
    bad[:, 7], bad[1, 299] = True, True
    assert torch.equal(torch.isnan(c), bad) and float(c[3, 140]) == float("inf")
    blocks = torch.zeros(n, s.shape[1], dtype=torch.bool, device="cuda")
    blocks[:, 0], blocks[3, 1], blocks[1, 2] = True, True, True
    assert torch.equal(s.view(torch.uint8) == 255, blocks)
    assert torch.equal(q.view(torch.uint8) == 0x7F, blocks.repeat_interleave(128, 1)[:, :m])


def test_ends_of_the_functions(b2):
    """Infinite, huge, zero and NaN z come from the bias; values and derivatives have their limits."""
    z = torch.tensor([float("-inf"), float("inf"), float("nan"), 0.0, -0.0, -1e30, 1e30, -88.0, 88.0, -1e4, 12.0, -14.0] + [1.0] * 4)
    m, n = z.numel(), 3
    a = torch.zeros(m, 128, device="cuda").to(F8)
    s = torch.full((m, 1), 127, dtype=torch.uint8, device="cuda").view(E8)
    for kind in ffn.ACTS:
        code = getattr(b2, "ACT_" + kind.upper())
        c = torch.empty(n, m, device="cuda")
        b2.b2_gemm_f8_act("T", "N", m, n, 128, 1.0, a, 128, s, 1, 1, a, 128, s, 1, 1, code, z.cuda(), None, m, None, m, c, m, None, m, None, 1)
        want = ffn.act(np64(z), kind)
        assert np.allclose(np64(c), np.broadcast_to(want, (n, m)), rtol=2.0**-20, atol=2.0**-20, equal_nan=True), kind
        dy, dz = torch.ones(n, m, device="cuda"), torch.empty(n, m, device="cuda")
        b2.b2_act_backward(m, n, code, dy, m, z.cuda().repeat(n, 1), m, dz, m, None, m, None, 1, None)
        want = ffn.act_slope(np64(z), kind)
        assert np.allclose(np64(dz), np.broadcast_to(want, (n, m)), rtol=0, atol=2.0**-18, equal_nan=True), kind


# ---- the activation's backward pass ------------------------------------------------------------------------------------
BACKWARD = [(1, 1, 0), (8, 3, 0), (127, 2, 0), (128, 64, 0), (129, 65, 3), (1003, 33, 24), (1003, 200, 0), (256, 9000, 0), (4096, 300, 8), (16390, 70, 2), (40000, 3, 0), (300, 8193, 4)]


@pytest.mark.parametrize("act,parts", [("gelu", "zqb"), ("none", "qb"), ("silu", "z"), ("gelu_tanh", "b"), ("relu", "zq")])
@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("d,t,pad", BACKWARD)
def test_backward(b2, d, t, pad, dt, act, parts):
    g = torch.Generator().manual_seed(d + t)
    dy, z = torch.randn(t, d, generator=g).to(dt), (2 * torch.randn(t, d, generator=g)).to(dt)
    ld, nb, offset = d + pad, -(-d // 128), pad % 2
    dz, q, s = buffer(t, ld, dt, offset) if "z" in parts else None, buffer(t, ld, F8, offset) if "q" in parts else None, buffer(t, nb + 1, E8) if "q" in parts else None
    db = torch.full((d,), float("nan"), device="cuda") if "b" in parts else None
    nws = b2.b2_act_backward_workspace_bytes(d, t)
    ws = torch.full((nws,), 0xFF, dtype=torch.uint8, device="cuda") if nws else None
    b2.b2_act_backward(d, t, getattr(b2, "ACT_" + act.upper()), stored(dy, ld, offset), ld, None if act == "none" else stored(z, ld, offset), ld, dz, ld, q, ld, s, nb + 1, db, ws)
    v = np64(dy) * ffn.act_slope(np64(z), act)
    e = np.abs(np64(dy)) * (0 if act in ("none", "relu") else 2.0**-18) + U * np.abs(v)
    if dz is not None:
        assert np.all(np.abs(np64(rows_of(dz, t, d, ld)) - v) <= e + HALF[dt] * (np.abs(v) + e))
    if q is not None:
        check_quantised(rows_of(q, t, d, ld), rows_of(s, t, nb, nb + 1), v, e)
    if db is not None:
        assert np.all(np.abs(np64(db) - v.sum(0)) <= e.sum(0) + (t + 4) * U * np.abs(v).sum(0))


@pytest.mark.parametrize("act", ffn.ACTS)
def test_backward_is_the_difference_of_the_forward(b2, act):
    """dz against (act(z + h) - act(z - h)) / 2h of the products' own epilogue, fp32.  h = 2^-6: the third derivative's part is below h^2 / 6 * 1.5 (none of
    these functions' third derivatives exceeds 1.5 in magnitude, away from relu's corner), both values are within 2^-20 * 8 (|z| < 8) of the function."""
    m, n, h = 260, 9, 2.0**-6
    z = torch.randint(-256, 256, (m,)).float() / 64 + 2.0**-5  # z + h, z - h and their difference are exact; never 0
    a = torch.zeros(m, 128, device="cuda").to(F8)
    s = torch.full((m, 1), 127, dtype=torch.uint8, device="cuda").view(E8)
    code = getattr(b2, "ACT_" + act.upper())

    def forward(at):
        c = torch.empty(n, m, device="cuda")
        b2.b2_gemm_f8_act("T", "N", m, n, 128, 1.0, a, 128, s, 1, 1, a, 128, s, 1, 1, code, at.cuda(), None, m, None, m, c, m, None, m, None, 1)
        return np64(c)

    z = torch.where(z.abs() <= h, 0.5, z)
    dz = torch.empty(n, m, device="cuda")
    b2.b2_act_backward(m, n, code, torch.ones(n, m, device="cuda"), m, z.cuda().repeat(n, 1), m, dz, m, None, m, None, 1, None)
    diff = (forward(z + h) - forward(z - h)) / (2 * h)
    assert np.max(np.abs(diff - np64(dz))) <= h * h / 6 * 1.5 + 2 * 8 * 2.0**-20 / (2 * h) + 2.0**-18


def test_backward_in_place_and_without_tokens(b2):
    d, t = 300, 90
    dy, z = torch.randn(t, d, device="cuda"), torch.randn(t, d, device="cuda")
    outs = []
    for where in (None, "dy", "z"):
        y, w = dy.clone(), z.clone()
        dz = {None: torch.empty_like(y), "dy": y, "z": w}[where]
        db = torch.empty(d, device="cuda")
        ws = torch.empty(b2.b2_act_backward_workspace_bytes(d, t), dtype=torch.uint8, device="cuda")
        b2.b2_act_backward(d, t, b2.ACT_GELU, y, d, w, d, dz, d, None, d, None, 1, db, ws)
        outs.append((dz.clone(), db))
    assert all(torch.equal(o[i], outs[0][i]) for o in outs for i in (0, 1))
    db = torch.full((d,), float("nan"), device="cuda")
    b2.b2_act_backward(d, 0, b2.ACT_NONE, dy, d, None, d, None, d, None, d, None, 3, db)
    assert bool((db == 0).all())


def test_backward_not_finite(b2):
    """What is not finite stays in its feature's sum and its block."""
    d, t = 300, 100
    dy, z = torch.ones(t, d, device="cuda"), torch.ones(t, d, device="cuda")
    dy[50, 10], z[70, 200] = float("inf"), float("nan")
    dz, q, s, db = torch.empty(t, d, device="cuda"), torch.empty(t, d, dtype=F8, device="cuda"), torch.empty(t, 3, dtype=E8, device="cuda"), torch.empty(d, device="cuda")
    ws = torch.empty(b2.b2_act_backward_workspace_bytes(d, t), dtype=torch.uint8, device="cuda")
    b2.b2_act_backward(d, t, b2.ACT_SILU, dy, d, z, d, dz, d, q, d, s, 3, db, ws)
    nan = (s.view(torch.uint8) == 255).nonzero().tolist()
    assert nan == [[50, 0], [70, 1]] and float(db[10]) == float("inf") and bool(torch.isnan(db[200])) and int(torch.isfinite(db).sum()) == d - 2


# ---- all of them ----------------------------------------------------------------------------------------------------
def block_step(b2, st):
    """Forward and backward pass of up, activation, down with residual, from and to the same buffers."""
    t, d, f = st["t"], st["d"], st["f"]
    b2.b2_quant_f8(d, t, 1, st["x"], d, st["xq"], d, st["xs"], st["xs"].shape[1])
    b2.b2_gemm_f8_act("T", "N", f, t, d, 1.0, st["w1"], d, st["s1"], st["s1"].shape[1], 128, st["xq"], d, st["xs"], st["xs"].shape[1], 1, b2.ACT_GELU, st["b1"], st["z"], f, None, f, None, f,
                      st["aq"], f, st["as"], st["as"].shape[1])
    b2.b2_gemm_f8_act("T", "N", d, t, f, 1.0, st["w2"], f, st["s2"], st["s2"].shape[1], 128, st["aq"], f, st["as"], st["as"].shape[1], 1, b2.ACT_NONE, st["b2"], None, d, st["x"], d, st["y"], d,
                      None, d, None, 1)
    b2.b2_act_backward(d, t, b2.ACT_NONE, st["dy"], d, None, d, None, d, st["dq"], d, st["ds"], st["ds"].shape[1], st["db2"], st["ws"])
    b2.b2_gemm_f8_act("N", "N", f, t, d, 1.0, st["w2"], f, st["s2"], st["s2"].shape[1], 128, st["dq"], d, st["ds"], st["ds"].shape[1], 1, b2.ACT_GELU | b2.ACT_GRADIENT, None, st["z"], f, None, f,
                      st["dz"], f, st["zq"], f, st["zs"], st["zs"].shape[1])
    b2.b2_act_backward(f, t, b2.ACT_NONE, st["dz"], f, None, f, None, f, None, f, None, 1, st["db1"], st["ws"])


def block_state(t, d, f, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    nd, nf = -(-d // 128), -(-f // 128)
    e8 = lambda *n: torch.empty(*n, dtype=E8, device="cuda")  # noqa: E731
    q8 = lambda *n: torch.empty(*n, dtype=F8, device="cuda")  # noqa: E731
    bf = lambda *n: torch.empty(*n, dtype=BF, device="cuda")  # noqa: E731
    st = {"t": t, "d": d, "f": f, "x": torch.randn(t, d, device="cuda", generator=g).bfloat16(), "dy": torch.randn(t, d, device="cuda", generator=g).bfloat16(),
          "w1": (0.5 * torch.randn(f, d, device="cuda", generator=g)).to(F8), "w2": (0.5 * torch.randn(d, f, device="cuda", generator=g)).to(F8),
          "s1": torch.full((nf, nd), 124, dtype=torch.uint8, device="cuda").view(E8), "s2": torch.full((nd, nf), 124, dtype=torch.uint8, device="cuda").view(E8),
          "b1": torch.randn(f, device="cuda", generator=g), "b2": torch.randn(d, device="cuda", generator=g), "xq": q8(t, d), "xs": e8(t, nd), "z": bf(t, f), "aq": q8(t, f), "as": e8(t, nf),
          "y": bf(t, d), "dq": q8(t, d), "ds": e8(t, nd), "dz": bf(t, f), "zq": q8(t, f), "zs": e8(t, nf), "db1": torch.empty(f, device="cuda"), "db2": torch.empty(d, device="cuda"),
          "ws": torch.empty(1 << 20, dtype=torch.uint8, device="cuda")}
    return st


RESULTS = ("z", "aq", "as", "y", "dz", "zq", "zs", "db1", "db2")


def test_together_on_a_stream_and_captured(b2):
    """The same bits directly, on another stream while two states are under way, and from a replayed graph with new inputs."""
    sizes = (200, 256, 528)
    want = []
    for seed in (1, 2):
        st = block_state(*sizes, seed)
        block_step(b2, st)
        want.append({k: st[k].clone().view(torch.uint8) for k in RESULTS})
    same = lambda st, w: all(torch.equal(st[k].view(torch.uint8), w[k]) for k in RESULTS)  # noqa: E731
    states = [block_state(*sizes, s) for s in (1, 2)]
    streams = [torch.cuda.Stream() for _ in states]
    torch.cuda.synchronize()
    for st, stream in zip(states, streams):
        with torch.cuda.stream(stream):
            for _ in range(3):
                block_step(b2, st)
    torch.cuda.synchronize()
    assert same(states[0], want[0]) and same(states[1], want[1])
    st, other = block_state(*sizes, 1), block_state(*sizes, 2)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        block_step(b2, st)
    graph.replay()
    torch.cuda.synchronize()
    assert same(st, want[0])
    for k in ("x", "dy", "w1", "w2", "b1", "b2"):
        st[k].view(torch.uint8).copy_(other[k].view(torch.uint8))
    graph.replay()
    torch.cuda.synchronize()
    assert same(st, want[1]) and b2.b2_device_status() == 0


def test_columns_far_apart(b2):
    """Offsets beyond 32 bits in Z, R, C and Q, and in the backward pass."""
    m, n, k, ld = 136, 1100, 128, 4_000_016
    a, sa, b, sb = plain_operands(m, n, k)
    bias = torch.randn(m, device="cuda")
    big, small = torch.empty(n * ld, dtype=torch.uint8, device="cuda").view(F8), torch.empty(n, m, dtype=F8, device="cuda")
    s, s2 = torch.empty(n, 2, dtype=E8, device="cuda"), torch.empty(n, 2, dtype=E8, device="cuda")
    far, near = torch.empty(n * ld, dtype=BF, device="cuda"), torch.empty(n, m, dtype=BF, device="cuda")
    for c, ldc, q, ldq, sc in ((far, ld, big, ld, s), (near, m, small, m, s2)):
        b2.b2_gemm_f8_act("T", "N", m, n, k, 0.25, a, k, sa, 1, 128, b, k, sb, 1, 1, b2.ACT_SILU, bias, None, m, None, m, c, ldc, q, ldq, sc, 2)
    assert torch.equal(far.view(n, ld)[:, :m], near) and torch.equal(big.view(torch.uint8).view(n, ld)[:, :m], small.view(torch.uint8)) and torch.equal(s.view(torch.uint8), s2.view(torch.uint8))
    db, db2 = torch.empty(m, device="cuda"), torch.empty(m, device="cuda")
    ws = torch.empty(b2.b2_act_backward_workspace_bytes(m, n), dtype=torch.uint8, device="cuda")
    b2.b2_act_backward(m, n, b2.ACT_GELU, far, ld, far, ld, far, ld, None, m, None, 2, db, ws)
    out = torch.empty_like(near)
    b2.b2_act_backward(m, n, b2.ACT_GELU, near, m, near, m, out, m, None, m, None, 2, db2, ws)
    assert torch.equal(far.view(n, ld)[:, :m], out) and torch.equal(db, db2)
