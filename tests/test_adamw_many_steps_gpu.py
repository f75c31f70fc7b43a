"""Fifty steps with moments in 8 bits on the GPU and by their definition in 64 bits, with the same random bits: the same numbers, but for those of an element whose fraction once was within its
error of the bits' border (2^-20 * 8 of them a step in the mean, see test_adamw_gpu.py; it then goes its own way, and its block's scale, where it is the largest, with it)."""
import numpy as np
import pytest
import torch

from oracle import f8
from test_adamw_many_steps import B1, B2, N, follow

pytestmark = pytest.mark.gpu
F8, E8 = torch.float8_e4m3fn, torch.float8_e8m0fnu


@pytest.mark.parametrize("offset", [0, 1])
def test_fifty_steps(b2, offset):
    g = np.random.default_rng(2)
    size = np.repeat(np.exp(g.standard_normal(N // 16)), 16)
    grads = [(size * (0.3 + g.standard_normal(N))).astype(np.float32) for _ in range(50)]
    zeros = lambda: torch.zeros(N + offset, dtype=torch.uint8, device="cuda")[offset:].view(F8)  # noqa: E731
    ones = lambda: torch.full((N // 128,), 127, dtype=torch.uint8, device="cuda").view(E8)  # noqa: E731
    p, m, v, sm, sv = torch.zeros(N + offset, device="cuda")[offset:], zeros(), zeros(), ones(), ones()
    for t, (gr, (m8, r8, *_)) in enumerate(zip(grads, follow(x.astype(np.float64) for x in grads)), 1):
        x = torch.empty(N + offset, device="cuda")[offset:].copy_(torch.from_numpy(gr))
        b2.b2_adamw([p], [x], [m], [v], [sm], [sv], 1e-3, B1, B2, 1e-8, 0.0, t, 5)
        for q, s, want in ((m, sm, m8), (v, sv, r8)):
            got = q.float().cpu().double().numpy() * np.repeat(f8.e8m0(s.view(torch.uint8).cpu().numpy()), 128)
            off = int((got != want).sum())
            assert off <= 3 + t * 20e-6 * N * (1 + 1 / (1 - B1)), (t, off)  # what fell to another number stays there for some steps
