"""Many steps with moments in 8 bits, by the definition (oracle/ffn.py): what random roundings do to the moments over time, beside moments that are never rounded.

m is linear in what was stored: its mean stays right.  Its spread: a rounding between two e4m3 numbers a distance h apart has a variance of at most h^2/4, h at most 2^-3 of the number, so at most 2^-8 of its
square, and 1 / (1 - beta1^2) of that remain of all steps.  The root is rounded without bias, its square then is not: v gains the variance, at most 2^-8 of itself a step, of which
beta2 / (1 - beta2) remain; numbers below 2^-6 of their block's scale have larger distances and are left out of the means."""
import numpy as np

from oracle import ffn

B1, B2 = 0.9, 0.95
N, STEPS = 4096, 200


def follow(grads, seed=5):
    """Stored (m, r) after every step, and those that were never rounded."""
    m8 = r8 = m = v = np.zeros(N)
    for t, g in enumerate(grads, 1):
        _, m8, v8 = ffn.adamw(0.0, g, m8, r8 * r8, 1e-3, B1, B2, 1e-8, 0.0, t)
        _, m, v = ffn.adamw(0.0, g, m, v, 1e-3, B1, B2, 1e-8, 0.0, t)
        bits = ffn.random_bits(np.arange(N), seed, t)
        (qm, sm), (qr, sr) = ffn.quantise_at_random(m8, bits[0], False), ffn.quantise_at_random(np.sqrt(v8), bits[1], True)
        m8, r8 = qm * np.repeat(sm, 128), qr * np.repeat(sr, 128)
        yield m8, r8, m, v, np.repeat(sr, 128)


def test_moments_over_many_steps():
    g = np.random.default_rng(1)
    size = np.repeat(np.exp(g.standard_normal(N // 16)), 16)
    for m8, r8, m, v, scale in follow(size * (0.3 + g.standard_normal(N)) for _ in range(STEPS)):
        pass
    root, fine = np.sqrt(v), r8 > scale * 2.0**-6
    assert fine.mean() > 0.9
    spread = 2.0**-4 * (1 / (1 - B1 * B1)) ** 0.5  # of m, relative to the largest that it has been lately
    off = (m8 - m)[fine] / root[fine]
    assert abs(off.mean()) < 5 * off.std() / off.size**0.5 and off.std() < 2 * spread
    gain = (r8 * r8 / v)[fine] - 1
    error = 5 * gain.std() / gain.size**0.5
    assert -error < gain.mean() < 2.0**-8 * B2 / (1 - B2) + error
