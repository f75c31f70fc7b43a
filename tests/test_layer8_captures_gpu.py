"""One 8-bit layer in several captured graphs: every call reads an 8-bit weight that has been made and still is, whichever runs first."""
import pytest
import torch

from paper_1611_08035_b200 import layer8

pytestmark = pytest.mark.gpu


def make():
    torch.manual_seed(7)
    layer = layer8.NormLinear8(256, 512)
    return layer, torch.randn(40, 256, device="cuda").bfloat16()


def test_captures_after_a_change(b2):
    """Both graphs make an 8-bit weight of their own, eager calls theirs: the second graph runs last but one, the first one last."""
    layer, x = make()
    with torch.no_grad():
        layer(x)
        layer.weight.mul_(2.0)
        graphs, results = [torch.cuda.CUDAGraph() for _ in range(2)], []
        torch.cuda.synchronize()
        for graph in graphs:
            with torch.cuda.graph(graph):
                results.append(layer(x)[0])
        want, _ = layer(x)
        fresh = layer8.NormLinear8(256, 512)
        fresh.load_state_dict(layer.state_dict())
        assert torch.equal(want, fresh(x)[0])
        for at in (1, 0):
            graphs[at].replay()
            torch.cuda.synchronize()
            assert torch.equal(results[at], want)
    assert b2.b2_device_status() == 0


def test_what_a_graph_reads_stays(b2):
    layer, x = make()
    with torch.no_grad():
        want, _ = layer(x)
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            y, _ = layer(x)
        layer.weight.mul_(2.0)
        layer(x)
        filler = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in 64 * (512 * 256, 8)]  # where the freed weight was
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)
        del filler


def test_a_captured_training_step(b2):
    layer, x = make()
    dy, side = torch.randn(40, 512, device="cuda").bfloat16(), torch.cuda.Stream()

    def step():
        layer.zero_grad()
        layer.requantise()
        layer(x)[0].backward(dy)

    step()
    want = [p.grad.clone() for p in layer.parameters()]
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        step()
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=side):
            step()
    for p in layer.parameters():
        p.grad.fill_(float("nan"))
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p.grad, w) for p, w in zip(layer.parameters(), want)) and b2.b2_device_status() == 0


def test_graphed_callable(b2):
    """torch's own way to capture both passes, whose warm-up's graph is alive meanwhile: gradients are handed out, none is added up."""
    layer, x = make()
    x.requires_grad_()
    dy = torch.randn(40, 512, device="cuda").bfloat16()

    def passes(f):
        x.grad = None
        layer.zero_grad()
        y, h = f(x)
        torch.autograd.backward([y, h], [dy, dy[:, :256].contiguous()])
        return [y.detach(), h.detach(), x.grad, *(p.grad for p in layer.parameters())]

    want = passes(layer)
    graphed = torch.cuda.make_graphed_callables(layer, (x.detach().clone().requires_grad_(),))
    for _ in range(2):
        assert all(torch.equal(a, b) for a, b in zip(passes(graphed), want))
    assert b2.b2_device_status() == 0


def test_beside_living_graphs(b2):
    """Of another stream: captured as if it were not there.  Of the default stream: refused, and what was captured of the step ends as any step that failed."""
    layer, x = make()
    dy, sides = torch.randn(40, 512, device="cuda").bfloat16(), [torch.cuda.Stream() for _ in range(2)]
    layer(x)[0].backward(dy)
    want = [p.grad.clone() for p in layer.parameters()]
    layer.zero_grad()
    torch.cuda.synchronize()
    with torch.cuda.stream(sides[0]):
        alive = layer(x)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=sides[1]):
        layer(x)[0].backward(dy)
    for p in layer.parameters():
        p.grad.fill_(float("nan"))
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p.grad, w) for p, w in zip(layer.parameters(), want))
    del alive, graph
    layer.zero_grad()
    alive = layer(x)
    torch.cuda.synchronize()
    with pytest.raises(RuntimeError, match="alive"):
        with torch.cuda.graph(torch.cuda.CUDAGraph(), stream=sides[1]):
            layer(x)[0].backward(dy)
    assert all(p.grad is None for p in layer.parameters())
    del alive
    layer(x)[0].backward(dy)
    assert all(torch.equal(p.grad, w) for p, w in zip(layer.parameters(), want)) and b2.b2_device_status() == 0
