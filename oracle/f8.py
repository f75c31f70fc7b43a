"""The 8-bit operators by their definitions, in 64 bits with numpy: what b2_quant_f8, b2_rmsnorm_f8, b2_rmsnorm_backward,
b2_gemm_f8 and b2_wgrad_f8 compute.  Shares no code with the CUDA library.

Matrices are numpy arrays [tokens][features] (the library's column-major storage read row by row)."""
from __future__ import annotations

import numpy as np

BLOCK = 128


def _e4m3_table() -> np.ndarray:
    """Value of every byte: 1 sign, 4 exponent (bias 7), 3 mantissa bits; exponent 0 is subnormal; 0x7f and 0xff are NaN."""
    out = np.empty(256)
    for b in range(256):
        sign, e, m = -1.0 if b & 0x80 else 1.0, (b >> 3) & 15, b & 7
        out[b] = np.nan if (e == 15 and m == 7) else sign * (m / 8.0 * 2.0**-6 if e == 0 else (1 + m / 8.0) * 2.0 ** (e - 7))
    return out


E4M3 = _e4m3_table()


def e8m0(byte: np.ndarray) -> np.ndarray:
    """Value of scale bytes: 2^(b - 127), 255 is NaN."""
    b = np.asarray(byte).astype(np.int64)
    return np.where(b == 255, np.nan, np.ldexp(1.0, np.minimum(b, 254) - 127))


def to_e4m3(v: np.ndarray) -> np.ndarray:
    """Bytes of the nearest e4m3 numbers, ties to the even mantissa; |v| <= 464 (nothing saturates), NaN to 0x7f."""
    pos = E4M3[:127]
    a = np.abs(v)
    hi = np.clip(np.searchsorted(pos, a, side="left"), 1, 126)
    lo = hi - 1
    d_lo, d_hi = a - pos[lo], pos[hi] - a
    pick = np.where((d_hi < d_lo) | ((d_hi == d_lo) & (hi % 2 == 0)), hi, lo)
    return np.where(np.isnan(v), 0x7F, pick | (np.signbit(v).astype(np.int64) << 7)).astype(np.uint8)


def scale_byte(amax: float) -> int:
    """The smallest power of two that brings amax to 448 or below, by trying them."""
    if not np.isfinite(amax):
        return 255
    if amax == 0:
        return 127
    b = 0
    while amax / 2.0 ** (b - 127) > 448.0:
        b += 1
    return b


def quantise(x: np.ndarray, block: int = 1):
    """Bytes q [t][d] and s [ceil(t/block)][ceil(d/128)] of x [t][d]."""
    t, d = x.shape
    q = np.zeros((t, d), np.uint8)
    s = np.zeros((-(-t // block), -(-d // BLOCK)), np.uint8)
    for i in range(s.shape[0]):
        for j in range(s.shape[1]):
            rows, cols = slice(i * block, (i + 1) * block), slice(j * BLOCK, (j + 1) * BLOCK)
            part = x[rows, cols].astype(np.float64)
            s[i, j] = scale_byte(np.max(np.abs(part)))
            q[rows, cols] = 0x7F if s[i, j] == 255 else to_e4m3(part / e8m0(s[i, j]))
    return q, s


def spread(s: np.ndarray, shape, block: int = 1) -> np.ndarray:
    """One scale per tile to one per element of an array [rows][summed index]."""
    return np.repeat(np.repeat(s, block, 0)[: shape[0]], BLOCK, 1)[:, : shape[1]]


def rmsnorm(x, r, w, eps):
    """(h, rstd, y) in 64 bits; r may be None."""
    h = x.astype(np.float64) + (0.0 if r is None else r.astype(np.float64))
    rstd = 1.0 / np.sqrt(np.mean(h * h, axis=1) + eps)
    return h, rstd, h * rstd[:, None] * w.astype(np.float64)


def rmsnorm_backward(dy, h, rstd, w, dh=None):
    """(dx, dw) in 64 bits; rstd is taken as given."""
    dy, xh = dy.astype(np.float64), h.astype(np.float64) * rstd.astype(np.float64)[:, None]
    g = dy * w.astype(np.float64)
    dx = rstd.astype(np.float64)[:, None] * (g - xh * np.mean(g * xh, axis=1, keepdims=True))
    return dx + (0.0 if dh is None else dh.astype(np.float64)), np.sum(dy * xh, axis=0)


def gemm(qa, sa, block_a, qb, sb, block_b):
    """sum_p a(i,p) b(j,p) and the sum of magnitudes, [n][m]; qa [m][k], qb [n][k] values, sa, sb [.][ceil(k/128)] values."""
    a, b = qa * spread(sa, qa.shape, block_a), qb * spread(sb, qb.shape, block_b)
    return b @ a.T, np.abs(b) @ np.abs(a).T


def wgrad(q, s, y):
    """sum_p x(p,i) y(p,j) and the sum of magnitudes, [n][m]; q [k][m], s [k][ceil(m/128)], y [k][n] values."""
    x = q * spread(s, q.shape)
    return y.T @ x, np.abs(y).T @ np.abs(x)
