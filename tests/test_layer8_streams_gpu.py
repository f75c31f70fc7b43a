"""One layer on two streams: whichever call makes its 8-bit weight, those of other streams read it when it is made, and its memory is not given away while one of them has yet to read
it.  What takes a stream long is a sleep on the device, a tenth of a second."""
import copy

import pytest
import torch

from paper_1611_08035_b200 import layer8

pytestmark = pytest.mark.gpu
LONG = 200_000_000  # clocks


def make():
    torch.manual_seed(8)
    layer = layer8.NormLinear8(256, 512)
    return layer, torch.randn(40, 256, device="cuda").bfloat16(), torch.cuda.Stream(), torch.cuda.Stream()


@pytest.mark.parametrize("explicit", [False, True])
def test_made_on_one_stream_and_read_on_another(b2, explicit):
    layer, x, a, b = make()
    with torch.no_grad():
        layer(x)
        layer.weight.mul_(2.0)
        torch.cuda.synchronize()  # the weight is there; its 8-bit form is not
        with torch.cuda.stream(a):
            torch.cuda._sleep(LONG)
            if explicit:
                layer.requantise()
            else:
                layer(x)
        with torch.cuda.stream(b):
            y, _ = layer(x)
        torch.cuda.synchronize()
        want, _ = copy.deepcopy(layer)(x)
        assert torch.equal(y, want) and b2.b2_device_status() == 0


def test_memory_that_another_stream_reads(b2):
    layer, x, a, b = make()
    with torch.no_grad(), torch.cuda.stream(a):
        layer.requantise()
        want, _ = layer(x)
        torch.cuda.synchronize()
        with torch.cuda.stream(b):
            torch.cuda._sleep(LONG)
            y, _ = layer(x)  # reads what was made on a, a tenth of a second from now
        layer.requantise()  # and a has another
        filler = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in 64 * (512 * 256, 8)]
        torch.cuda.synchronize()
        assert torch.equal(y, want)
        del filler
