"""A feed-forward block's operators by their definitions, in 64 bits with numpy: what b2_gemm_f8_act, b2_act_backward and b2_adamw compute.
Shares no code with the CUDA library."""
from __future__ import annotations

import math

import numpy as np

from . import f8

ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")
_erfc = np.vectorize(math.erfc, otypes=[np.float64])


def act(z: np.ndarray, kind: str) -> np.ndarray:
    with np.errstate(over="ignore", invalid="ignore"):
        if kind == "none":
            return z
        if kind == "relu":
            return np.where(z < 0, 0.0, z)
        if kind == "gelu":
            y = 0.5 * z * _erfc(-z / math.sqrt(2))
        elif kind == "silu":
            y = z / (1 + np.exp(-z))
        else:
            y = 0.5 * z * _erfc2(z)
        return np.where(z == -np.inf, 0.0, y)


def _erfc2(z):
    """1 + tanh of the tanh form's argument, without cancellation."""
    u = math.sqrt(2 / math.pi) * (z + 0.044715 * z**3)
    return 2 / (1 + np.exp(-2 * u))


def act_slope(z: np.ndarray, kind: str) -> np.ndarray:
    """The derivative; its limits where z is infinite."""
    with np.errstate(over="ignore", invalid="ignore"):
        if kind == "none":
            return np.ones_like(z)
        if kind == "relu":
            return np.where(np.isnan(z), np.nan, (z > 0).astype(np.float64))
        if kind == "gelu":
            y = 0.5 * _erfc(-z / math.sqrt(2)) + z * np.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
        elif kind == "silu":
            s = 1 / (1 + np.exp(-z))
            y = s + z * s / (1 + np.exp(z))
        else:
            u, du = math.sqrt(2 / math.pi) * (z + 0.044715 * z**3), math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z * z)
            s = 1 / (1 + np.exp(-2 * u))
            y = s + z * s / (1 + np.exp(2 * u)) * 2 * du
        return np.where(np.isinf(z), (z > 0).astype(np.float64), y)


LOW = 0xFFFFFFFF
GOLDEN = 0x9E3779B9


def fmix(x):
    """The finaliser of MurmurHash3 on unsigned 64-bit arrays that hold 32 bits."""
    x = np.asarray(x, np.uint64) & np.uint64(LOW)
    for shift, mul in ((16, 0x85EBCA6B), (13, 0xC2B2AE35)):
        x = ((x ^ (x >> np.uint64(shift))) * np.uint64(mul)) & np.uint64(LOW)
    return x ^ (x >> np.uint64(16))


def random_bits(e: np.ndarray, seed: int, step: int):
    """Twenty random bits for m and for the root of v of the elements numbered e."""
    key = int(fmix(int(fmix(int(fmix(seed & LOW)) ^ (seed >> 32 & LOW))) ^ (step & LOW)))
    e8 = np.asarray(e, np.uint64) >> np.uint64(3)
    h = fmix((e8 & np.uint64(LOW)) + fmix((e8 >> np.uint64(32)) + np.uint64(key)))
    j = (np.asarray(e, np.uint64) & np.uint64(7)) * np.uint64(GOLDEN)
    return tuple((((x + j) & np.uint64(LOW)) >> np.uint64(12)).astype(np.int64) for x in (h, fmix(h + np.uint64(GOLDEN))))


def at_random(y: np.ndarray, u: np.ndarray) -> np.ndarray:
    """y >= 0, at most 448: the e4m3 number below it, or the next one with probability of its distance; u is the twenty bits that decide."""
    with np.errstate(divide="ignore"):
        step = 2.0 ** (np.floor(np.log2(np.maximum(y, 2.0**-6))) - 3)
    return np.floor(y / step + u / 2.0**20) * step


def quantise_at_random(x: np.ndarray, u: np.ndarray, root: bool):
    """Values q and scales s of blocks of 128 of x; a root that is not 0 is at least 2^-9 of its scale."""
    q, s = np.empty_like(x), np.empty(-(-x.size // 128))
    for b in range(s.size):
        at = slice(128 * b, 128 * b + 128)
        s[b] = f8.e8m0(np.array(f8.scale_byte(np.max(np.abs(x[at])))))
        y = np.abs(x[at]) / s[b]
        r = at_random(y, u[at])
        q[at] = np.copysign(np.where(y > 0, np.maximum(r, 2.0**-9), r) if root else r, x[at])
    return q, s


def adamw(p, g, m, v, lr, beta1, beta2, eps, wd, step):
    """New (p, m, v) in 64 bits from 64-bit arrays."""
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    mh, vh = m / (1 - beta1**step), v / (1 - beta2**step)
    return p - lr * wd * p - lr * mh / (np.sqrt(vh) + eps), m, v
