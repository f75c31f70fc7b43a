"""Long lists of b2_adamw: overlaps are found wherever they are, without a GPU (every call is refused, or has nothing to do), and no entry point allocates memory on the host."""
import ctypes
import re
from pathlib import Path

import pytest

CSRC = Path(__file__).resolve().parent.parent / "paper_1611_08035_b200" / "csrc"


def test_sources_allocate_nothing():
    """The header promises it of every call.  calls.cpp is Python's, not the library's."""
    for f in sorted([*CSRC.glob("*.cu"), *CSRC.glob("*.cuh"), *CSRC.glob("*.h")]):
        text = re.sub(r'//[^\n]*|/\*.*?\*/|"[^"\n]*"', "", f.read_text(), flags=re.S)
        found = re.search(r"\bnew\b|\b[cm]alloc\s*\(|std::(vector|string|map|make_unique|unique_ptr|function)\b", text)
        assert not found, (f.name, found)


@pytest.mark.parametrize("count", [2, 33, 2048, 2049, 5000])
def test_overlaps_in_long_lists(b2, count):
    table = (b2._AdamwTensor * count)()
    far = 1 << 20

    def fill():
        for i in range(count):
            at = 4096 + (i * 7919 % count) * far  # in no order; never dereferenced
            table[i] = b2._AdamwTensor(at, 4096, 4096, 4096, None, None, 1000, b2._TYPES[b2._F32], b2._TYPES[b2._F32], 32, 0)

    def refused():
        d = ctypes.c_double
        return b2.lib().b2_adamw(table, count, d(0.1), d(0.9), d(0.99), d(1e-8), d(0.0), 1, 0, None, None, None, None)

    for i, j in {(0, count - 1), (count // 2, count // 2 - 1), (count - 1, count - 2), (min(2048, count - 1), 0)}:
        fill()
        table[i].param = table[j].param + 3996  # the other one's last number
        assert refused() == -1, (i, j)
