"""One feed-forward block in several captured graphs and on several streams: every call reads 8-bit weights that have been made, whichever runs first."""
import pytest
import torch

from paper_1611_08035_b200 import capture, ffn8

pytestmark = pytest.mark.gpu


def make():
    torch.manual_seed(7)
    block = ffn8.FeedForward8(256, 512)
    return block, torch.randn(40, 256, device="cuda").bfloat16()


def test_numbers_of_captures(b2):
    x = torch.zeros(1, device="cuda")
    numbers = []
    for _ in range(2):
        assert b2.b2_graph_capture_id(torch.cuda.current_stream().cuda_stream) == 0
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            numbers += [capture.capture_id(x), capture.capture_id(x)]
            x.add_(1)
    assert numbers[0] == numbers[1] != numbers[2] == numbers[3] and 0 not in numbers


def test_two_captures_after_a_change(b2):
    """Both graphs make 8-bit weights of their own: the second one runs first."""
    block, x = make()
    with torch.no_grad():
        block(x)
        block.up.mul_(2.0)
        graphs, results = [torch.cuda.CUDAGraph() for _ in range(2)], []
        torch.cuda.synchronize()
        for graph in graphs:
            with torch.cuda.graph(graph):
                results.append(block(x))
        graphs[1].replay()
        torch.cuda.synchronize()
        second = results[1].clone()
        want = block(x)
        graphs[0].replay()
        torch.cuda.synchronize()
        assert torch.equal(second, want) and torch.equal(results[0], want) and b2.b2_device_status() == 0


def test_a_capture_after_a_refused_one(b2):
    block, x = make()
    alive = block(x)
    with torch.no_grad():
        block.up.mul_(2.0)
    torch.cuda.synchronize()
    with pytest.raises(RuntimeError, match="alive"):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            block(x)
    del alive
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.no_grad(), torch.cuda.graph(graph):
        y = block(x)
    graph.replay()
    torch.cuda.synchronize()
    with torch.no_grad():
        assert torch.equal(y, block(x))


def test_graphed_callable(b2):
    """torch's own way to capture both passes, whose warm-up's graph is alive meanwhile."""
    block, x = make()
    x.requires_grad_()
    dy = torch.randn(40, 256, device="cuda").bfloat16()

    def passes(f):
        x.grad = None
        block.zero_grad()
        y = f(x)
        y.backward(dy)
        return [y.detach(), x.grad, *(p.grad for p in block.parameters())]

    want = passes(block)
    graphed = torch.cuda.make_graphed_callables(block, (x.detach().clone().requires_grad_(),))
    for _ in range(2):
        assert all(torch.equal(a, b) for a, b in zip(passes(graphed), want))
    assert b2.b2_device_status() == 0


def test_a_backward_pass_beside_a_graph_of_the_default_stream(b2):
    block, x = make()
    dy, side = torch.randn(40, 256, device="cuda").bfloat16(), torch.cuda.Stream()
    alive = block(x)
    alive.backward(dy, retain_graph=True)
    want = [p.grad for p in block.parameters()]
    block.zero_grad()
    torch.cuda.synchronize()
    with pytest.raises(RuntimeError, match="alive"):
        with torch.cuda.graph(torch.cuda.CUDAGraph(), stream=side):
            block(x).backward(dy)
    del alive
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        block(x).backward(dy)
    for p in block.parameters():
        p.grad.fill_(float("nan"))
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p.grad, w) for p, w in zip(block.parameters(), want)) and b2.b2_device_status() == 0
