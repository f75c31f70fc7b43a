"""One feed-forward block on two streams: whichever call makes its 8-bit weights, those of other streams read them when they are made, and their memory is not given away while one of
them has yet to read it.  What takes a stream long is a sleep on the device, a tenth of a second."""
import pytest
import torch

from paper_1611_08035_b200 import ffn8

pytestmark = pytest.mark.gpu
LONG = 200_000_000  # clocks


def make():
    torch.manual_seed(8)
    block = ffn8.FeedForward8(256, 512)
    return block, torch.randn(40, 256, device="cuda").bfloat16(), torch.cuda.Stream(), torch.cuda.Stream()


@pytest.mark.parametrize("explicit", [False, True])
def test_made_on_one_stream_and_read_on_another(b2, explicit):
    block, x, a, b = make()
    with torch.no_grad():
        block(x)
        block.up.mul_(2.0), block.down.mul_(0.5)
        torch.cuda.synchronize()  # the weights are there; their 8-bit forms are not
        with torch.cuda.stream(a):
            torch.cuda._sleep(LONG)
            if explicit:
                block.requantise()
            else:
                block(x)
        with torch.cuda.stream(b):
            y = block(x)
        torch.cuda.synchronize()
        want = ffn8.FeedForward8(256, 512)
        want.load_state_dict(block.state_dict())
        assert torch.equal(y, want(x))


def test_memory_that_another_stream_reads(b2):
    block, x, a, b = make()
    with torch.no_grad(), torch.cuda.stream(a):
        want = block(x)
        torch.cuda.synchronize()
        with torch.cuda.stream(b):
            torch.cuda._sleep(LONG)
            y = block(x)  # reads what was made on a, a tenth of a second from now
        block.requantise()  # and a has others
        filler = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in 8 * (512 * 256, 8)]
        torch.cuda.synchronize()
        assert torch.equal(y, want)
        del filler


def test_gradients_on_another_stream(b2):
    block, x, a, b = make()
    dy = torch.randn(40, 256, device="cuda").bfloat16()
    grads = []
    for streams in ((a, a), (a, b)):
        block.zero_grad()
        with torch.no_grad():
            block.up.add_(0.0)
        torch.cuda.synchronize()
        with torch.cuda.stream(streams[0]), torch.no_grad():
            torch.cuda._sleep(LONG)
            block(x)
        with torch.cuda.stream(streams[1]):
            block(x).backward(dy)
        torch.cuda.synchronize()
        grads.append([p.grad.clone() for p in block.parameters()])
    assert all(torch.equal(g, h) for g, h in zip(*grads)) and b2.b2_device_status() == 0


def test_captured_before_they_are_made(b2):
    """A capture that begins while the 8-bit weights are being made on another stream: the replay reads them, on any stream."""
    block, x, a, b = make()
    with torch.no_grad():
        want = block(x)
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.stream(a):
            torch.cuda._sleep(LONG)
            block.requantise()
        with torch.cuda.stream(b):
            graph.capture_begin()
            y = block(x)
            graph.capture_end()
            graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)


def test_two_streams_of_one_capture(b2):
    block, x, a, b = make()
    with torch.no_grad():
        want = block(x)
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=a):
            start = torch.cuda.Event()
            start.record(a)
            block.requantise()
            with torch.cuda.stream(b):
                b.wait_event(start)
                y = block(x)
            a.wait_stream(b)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)
