"""AdamW with moments in 8 bits at the ends of their range: aligned tensors, whose roots take a way of their own between 2^-50 and 2^64, hold the same bits as those that start anywhere, and
as the definition, with tolerances from test_adamw_gpu.py."""
import pytest
import torch

from test_adamw_gpu import call, check, placed, quantised, run

pytestmark = pytest.mark.gpu


def blocks(n, exponents, seed, zeros=0.3):
    """p, g, m, r with one power of two to each 128 elements; some gradients and roots, alone and together, are 0."""
    g = torch.Generator().manual_seed(seed)
    e = torch.tensor(exponents, dtype=torch.float64)[torch.randint(len(exponents), (n // 128,), generator=g)].repeat_interleave(128)
    size = torch.exp2(e)
    draw = lambda: torch.randn(n, generator=g, dtype=torch.float64) * size  # noqa: E731
    p, gr, m, r = torch.randn(n, generator=g).float(), draw().float(), draw().float(), (0.1 * size + draw().abs()).float()
    gr[torch.rand(n, generator=g) < zeros] = 0.0
    r[torch.rand(n, generator=g) < zeros] = 0.0
    return p, gr, m, r


def tensor(parts, offset):
    p, gr, m, r = parts
    (qm, sm), (qr, sr) = quantised(m), quantised(r)
    return {"p": placed(p, offset), "g": placed(gr, offset), "m": placed(qm, offset), "v": placed(qr, offset), "sm": sm.cuda(), "sv": sr.cuda()}


ENDS = {"small": [-56, -53, -51, -50, -49, -46], "ordinary": [-20, -10, 0, 10], "large": [40, 55, 60], "mixed": [-52, -50, -20, 0, 55]}


@pytest.mark.parametrize("kind", ENDS)
def test_against_the_definition(b2, kind):
    n = 1 << 15
    parts = blocks(n, ENDS[kind], 1)
    for offset in (0, 1):
        t = tensor(parts, offset)
        before, flips = {k: x.clone() for k, x in t.items()}, []
        call(b2, [t])
        check(before, t, 0, 10, 12345678901, flips=flips)
        off, total = (sum(x) for x in zip(*flips))
        assert off <= 3 + 20e-6 * total, (off, total)


@pytest.mark.parametrize("n", [1 << 16, 1 << 22])  # one piece of 256 to a warp, two
@pytest.mark.parametrize("kind", [*ENDS, "not finite"])
def test_aligned_and_other_tensors_agree(b2, kind, n):
    parts = blocks(n, ENDS.get(kind, [-50, 0, 60]), 2)
    if kind == "not finite":
        at = torch.randint(n, (n // 1000,), generator=torch.Generator().manual_seed(3))
        parts[1][at] = torch.tensor([float("inf"), float("-inf"), float("nan"), 3e38, -1e30, 2e19])[torch.arange(len(at)) % 6]  # the last ones' squares, too
    results = []
    for offset in (0, 1):
        t = tensor(parts, offset)
        call(b2, [t])
        results.append([t[k].view(torch.uint8).clone() for k in ("m", "v", "sm", "sv")] + [torch.isnan(t["p"])])
    assert all(torch.equal(a, b) for a, b in zip(*results))


def test_zero_roots_alone(b2):
    """Blocks of zeros beside others: nothing moves where there is no gradient, and a scale of zeros stays 1."""
    for n in (1 << 12, 1 << 22):
        t = tensor((torch.ones(n), torch.zeros(n), torch.zeros(n), torch.zeros(n)), 0)
        t["g"][n // 2 :] = 1.0
        call(b2, [t], wd=0.0)
        assert bool((t["p"][: n // 2] == 1.0).all()) and bool((t["p"][n // 2 :] < 1.0).all())
        assert bool((t["m"].view(torch.uint8)[: n // 2] == 0).all()) and bool((t["v"].view(torch.uint8)[: n // 2] == 0).all())
        assert bool((t["sm"].view(torch.uint8)[: n // 256] == 127).all()) and bool((t["sv"].view(torch.uint8)[: n // 256] == 127).all())


@pytest.mark.parametrize("bits", [8, 32])
def test_more_tensors_than_are_compared_at_once(b2, bits):
    run(b2, [1 + i * 37 % 150 for i in range(4500)], bits)
