"""The rule that splits k over clusters, by what it is for: time."""
import pytest
import torch

pytestmark = pytest.mark.gpu
F8, E8 = torch.float8_e4m3fn, torch.float8_e8m0fnu


def time_us(b2, m, n, k, scale):
    """One product among others, operands in turn so that they come from memory; the best of five."""
    copies = max(2, int(3e8 / (m * k)) + 1)
    ones = lambda *shape: torch.full(shape, 0x38, dtype=torch.uint8, device="cuda").view(F8)  # noqa: E731
    a, b = [ones(m, k) for _ in range(copies)], ones(n, k)
    scales = lambda rows: torch.full((rows, k // 128), 127, dtype=torch.uint8, device="cuda").view(E8)  # noqa: E731
    sa, sb = scales(-(-m // 128)), scales(n)
    if scale == "f32":
        sa, sb = sa.float(), sb.float()
    C = torch.empty(n, m, dtype=torch.bfloat16, device="cuda")
    graph = torch.cuda.CUDAGraph()
    run = lambda i: b2.b2_gemm_f8("T", "N", m, n, k, 1.0, a[i % copies], k, sa, k // 128, 128, b, k, sb, k // 128, 1, 0.0, C, m)  # noqa: E731
    run(0)
    with torch.cuda.graph(graph):
        for i in range(20):
            run(i)
    times = []
    for _ in range(6):
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        begin.record()
        graph.replay()
        end.record()
        end.synchronize()
        times.append(begin.elapsed_time(end) * 50)
    assert bool((C == k).all())
    return min(times[1:])


@pytest.mark.parametrize("scale", ["e8m0", "f32"])
@pytest.mark.parametrize("m,more", [(50304, 64000), (40001, 50304)])
def test_more_rows_take_no_less(b2, m, more, scale):
    """A vocabulary with a quarter more words is a quarter more work: where the smaller one takes longer, it was split for CTAs that do not fit."""
    for _ in range(3):  # the clock may change between the two
        few, many = time_us(b2, m, 64, 4096, scale), time_us(b2, more, 64, 4096, scale)
        if few <= 1.05 * many:
            return
    pytest.fail(f"{m} rows {few:.1f} us, {more} rows {many:.1f}")
