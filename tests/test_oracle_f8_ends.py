"""Where the largest numbers go when they are rounded to 8 bits (oracle/f8.py), as b2gemm.h says it."""
import numpy as np
import pytest

from oracle import f8


@pytest.mark.parametrize("v,back", [(1.9375, 2.0), (np.nextafter(1.9375, 0), 1.875), (np.finfo(np.float32).max / 2.0**127, 2.0), (255 / 128, 2.0), (1.75, 1.75)])
def test_largest_numbers(v, back):
    """A magnitude of 1.9375 * 2^127 or more (bf16's largest among them) comes back as 2^128, smaller ones as a number that bf16 holds."""
    q, s = f8.quantise(np.array([[v * 2.0**127]]))
    assert f8.E4M3[q[0, 0]] * f8.e8m0(s[0, 0]) == back * 2.0**127
