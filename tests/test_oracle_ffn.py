"""The definitions of the feed-forward block's operators: derivatives against differences, the random rounding against its expectation."""
import numpy as np
import pytest

from oracle import f8, ffn


@pytest.mark.parametrize("kind", ffn.ACTS)
def test_slope_is_the_derivative(kind):
    z = np.linspace(-9, 9, 401) + 1e-3
    h = 1e-6
    assert np.allclose((ffn.act(z + h, kind) - ffn.act(z - h, kind)) / (2 * h), ffn.act_slope(z, kind), rtol=0, atol=1e-8)


@pytest.mark.parametrize("kind", ffn.ACTS[1:])
def test_ends(kind):
    z = np.array([-np.inf, np.inf, np.nan, 0.0, -1e30, 1e30])
    assert np.array_equal(ffn.act(z, kind), [0, np.inf, np.nan, 0, 0, 1e30], equal_nan=True)
    assert np.array_equal(ffn.act_slope(z, kind)[[0, 1, 2, 4, 5]], [0, 1, np.nan, 0, 1], equal_nan=True)


def test_random_rounding_gives_neighbours_with_the_right_mean():
    y = np.array([0.0, 2.0**-9, 2.0**-11, 0.01, 2.0**-6, 0.3, 1.0, 17.1, 300.0, 447.9, 448.0])
    u = np.arange(0, 1 << 20, 16)
    got = ffn.at_random(y[:, None], u[None])
    pos = f8.E4M3[:127]
    assert np.isin(got, pos).all() and (np.abs(got - y[:, None]) < np.maximum(y[:, None] * 2.0**-3, 2.0**-9)).all()
    step = 2.0 ** (np.floor(np.log2(np.maximum(y, 2.0**-6))) - 3)
    assert (np.abs(got.mean(1) - y) <= step * 2.0**-16).all()  # u in steps of 16 of 2^20


def test_random_bits_look_random():
    a, b = ffn.random_bits(np.arange(1 << 16), 12345, 7)
    n = a.size
    for x in (a, b):
        assert 0 <= x.min() and x.max() < 1 << 20
        # mean of n uniform numbers: five standard deviations
        assert abs(x.mean() / 2**20 - 0.5) < 5 / np.sqrt(12 * n / 8)  # eight neighbours share a hash
    c = np.corrcoef(a, b)[0, 1]
    assert abs(c) < 5 / np.sqrt(n / 8)
    assert (ffn.random_bits(np.arange(64), 12345, 8)[0] != a[:64]).any() and (ffn.random_bits(np.arange(64), 12346, 7)[0] != a[:64]).any()


def test_numbers_past_32_bits_differ():
    e = np.arange(256, dtype=np.uint64)
    assert (ffn.random_bits(e, 1, 1)[0] != ffn.random_bits(e + np.uint64(1 << 35), 1, 1)[0]).any()


def test_adamw_is_its_textbook_form():
    rng = np.random.default_rng(0)
    p, m, v = rng.normal(size=50), np.zeros(50), np.zeros(50)
    w, b1, b2 = p.copy(), 0.9, 0.99
    gs = rng.normal(size=(4, 50))
    for t in range(1, 5):
        p, m, v = ffn.adamw(p, gs[t - 1], m, v, 1e-2, b1, b2, 1e-8, 0.1, t)
        mh = sum((1 - b1) * b1 ** (t - 1 - i) * gs[i] for i in range(t)) / (1 - b1**t)
        vh = sum((1 - b2) * b2 ** (t - 1 - i) * gs[i] ** 2 for i in range(t)) / (1 - b2**t)
        w = w * (1 - 1e-3) - 1e-2 * mh / (np.sqrt(vh) + 1e-8)
    assert np.allclose(p, w, rtol=1e-12, atol=0)
