"""Pins of the 8-bit oracle (oracle/f8.py): the number format, the quantisation rule, the norm's gradient."""
import numpy as np
import pytest
import torch

from oracle import f8


def test_e4m3_table_is_the_format():
    want = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).to(torch.float64).numpy()
    assert np.array_equal(f8.E4M3, want, equal_nan=True)
    assert f8.E4M3[126] == 448 and f8.E4M3[1] == 2.0**-9


def test_rounding_to_e4m3_matches_an_independent_conversion():
    rng = np.random.default_rng(0)
    v = np.concatenate([rng.uniform(-448, 448, 4000), rng.normal(size=4000) * 0.01, f8.E4M3[:127], -f8.E4M3[:127],
                        (f8.E4M3[:126] + f8.E4M3[1:127]) / 2])  # ties
    v = v.astype(np.float32)
    want = torch.from_numpy(v).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(f8.to_e4m3(v.astype(np.float64)), want)


def test_scale_rule():
    assert f8.scale_byte(0.0) == 127 and f8.scale_byte(448.0) == 127 and f8.scale_byte(np.nextafter(448.0, 500)) == 128
    assert f8.scale_byte(224.0) == 126 and f8.scale_byte(1.75) == 119 and f8.scale_byte(1.7500001) == 120
    assert f8.scale_byte(1e-44) == 0 and f8.scale_byte(np.inf) == 255 and f8.scale_byte(np.nan) == 255
    assert f8.scale_byte(float(np.finfo(np.float32).max)) == 247
    x = np.random.default_rng(1).normal(size=(5, 300)) * 10.0 ** np.arange(-2, 3)[:, None]
    q, s = f8.quantise(x)
    back = f8.E4M3[q] * f8.spread(f8.e8m0(s), x.shape)
    assert s.shape == (5, 3) and np.all(np.abs(back - x) <= np.maximum(np.abs(x) * 2.0**-4, f8.spread(f8.e8m0(s), x.shape) * 2.0**-10))


@pytest.mark.parametrize("with_residual_gradient", [False, True])
def test_norm_gradient_against_differences(with_residual_gradient):
    """d/dx and d/dw of sum(dy*y) + sum(dh*h) by central differences in 64 bits."""
    rng = np.random.default_rng(2)
    t, d, eps = 3, 37, 1e-3
    x, w, dy = rng.normal(size=(t, d)), rng.normal(size=d), rng.normal(size=(t, d))
    dh = rng.normal(size=(t, d)) if with_residual_gradient else None

    def loss(x, w):
        h, _, y = f8.rmsnorm(x, None, w, eps)
        return np.sum(dy * y) + (0.0 if dh is None else np.sum(dh * h))

    h, rstd, _ = f8.rmsnorm(x, None, w, eps)
    dx, dw = f8.rmsnorm_backward(dy, h, rstd, w, dh)
    step = 1e-5
    for _ in range(20):
        i, j = rng.integers(t), rng.integers(d)
        e = np.zeros((t, d))
        e[i, j] = step
        assert abs((loss(x + e, w) - loss(x - e, w)) / (2 * step) - dx[i, j]) < 1e-7
        assert abs((loss(x, w + e[i]) - loss(x, w - e[i])) / (2 * step) - dw[j]) < 1e-7


def test_products_against_explicit_sums():
    rng = np.random.default_rng(3)
    m, n, k = 130, 3, 257
    qa, qb = rng.integers(-4, 5, (m, k)).astype(float), rng.integers(-4, 5, (n, k)).astype(float)
    sa, sb = 2.0 ** rng.integers(-2, 3, (2, 3)), 2.0 ** rng.integers(-2, 3, (n, 3))
    got, mag = f8.gemm(qa, sa, 128, qb, sb, 1)
    for i, j in ((0, 0), (127, 1), (128, 2), (129, 0)):
        want = sum(qa[i, p] * sa[i // 128, p // 128] * qb[j, p] * sb[j, p // 128] for p in range(k))
        assert got[j, i] == want and mag[j, i] >= abs(want)
    y = rng.integers(-4, 5, (n, 5)).astype(float)
    q, s = rng.integers(-4, 5, (n, 130)).astype(float), 2.0 ** rng.integers(-2, 3, (n, 2))
    got, _ = f8.wgrad(q, s, y)
    assert got[4, 129] == sum(q[p, 129] * s[p, 1] * y[p, 4] for p in range(n))
