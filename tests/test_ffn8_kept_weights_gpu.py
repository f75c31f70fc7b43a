"""8-bit weights that a captured graph reads are kept while the graph lives, once, and no longer."""
import gc
import time
import weakref

import pytest
import torch

from paper_1611_08035_b200 import ffn8

pytestmark = pytest.mark.gpu


def make():
    torch.manual_seed(9)
    block = ffn8.FeedForward8(256, 512)
    return block, torch.randn(40, 256, device="cuda").bfloat16()


def captured(block, x):
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        y = block(x)
        block(x)
    return graph, y


def gone(reference):
    """Whether it is let go within some seconds: CUDA tells of a destroyed graph from a thread of its own."""
    for _ in range(100):
        gc.collect()
        if reference() is None:
            return True
        time.sleep(0.05)
    return False


def test_kept_while_the_graph_lives(b2):
    block, x = make()
    with torch.no_grad():
        want = block(x)
        weights = weakref.ref(block._quantised["up"][0][0])
        graph, y = captured(block, x)
        assert len(block._captured) == 1
        for _ in range(3):
            block.up.mul_(2.0)
            block(x)
        assert weights() is not None
        filler = [torch.full((512 * 256,), 255, dtype=torch.uint8, device="cuda") for _ in range(8)]
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want) and len(block._captured) == 1
        del graph, y, filler
        torch.cuda.synchronize()

        def asked():
            block._let_go()
            return weights()

        assert gone(asked) and not block._captured


def test_many_graphs(b2):
    """One after the other, each with weights of its own."""
    block, x = make()
    with torch.no_grad():
        block(x)
        for _ in range(5):
            graph, y = captured(block, x)
            graph.replay()
            block.requantise()
        graph.reset()
        del graph, y
        torch.cuda.synchronize()
        for _ in range(100):
            block._let_go()
            if not block._captured:
                break
            time.sleep(0.05)
        assert not block._captured


def test_places_of_watches_come_back(b2):
    stream = torch.cuda.current_stream().cuda_stream
    with pytest.raises(b2.B2Error):
        b2.b2_graph_watch(stream)  # no capture
    x = torch.zeros(8, device="cuda")
    for ask in (False, True):
        for _ in range(3):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                watches = [b2.b2_graph_watch(torch.cuda.current_stream().cuda_stream) for _ in range(2000)]
                x.add_(1)
            assert len(set(watches)) == 2000 and not any(b2.b2_graph_gone(w) for w in watches)
            if not ask:
                for w in watches:
                    b2.b2_graph_unwatch(w)
            del graph
            if ask:
                assert any(all(b2.b2_graph_gone(w) for w in watches) or time.sleep(0.05) for _ in range(100))
                for w in watches:
                    b2.b2_graph_unwatch(w)
            else:
                time.sleep(0.5)
