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


def test_a_capture_beside_a_living_graph_is_refused(b2):
    layer, x = make()
    alive = layer(x)  # both results, each of which keeps the graph
    torch.cuda.synchronize()
    with pytest.raises(RuntimeError, match="alive"):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            layer(x)
    alive[0].float().sum().backward()
    del alive
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
