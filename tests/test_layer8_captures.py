"""The 8-bit layer in several captures, without a GPU: captures are told apart by their numbers, the operators are test_layer8.py's stand-in."""
import copy

import pytest
import torch

from paper_1611_08035_b200 import layer8
from test_layer8 import make, ops  # noqa: F401


@pytest.fixture
def capture(monkeypatch):
    """The number of the capture that calls go into; 0: none."""
    now = [0]
    monkeypatch.setattr(layer8, "capturing", lambda x: now[0] != 0, raising=False)
    monkeypatch.setattr(layer8, "capture_id", lambda x: now[0], raising=False)
    return now


def test_what_one_capture_made_is_not_another_ones(ops, capture):  # noqa: F811
    layer, x, r = make()
    made = lambda: ops.calls.count("quant")  # noqa: E731
    with torch.no_grad():
        capture[0] = 5
        layer(x, r), layer(x, r)
        assert made() == 1
        capture[0] = 6  # whose graph may run before the other's
        layer(x, r), layer(x, r)
        assert made() == 2
        capture[0] = 0  # before either has run
        layer(x, r)
        assert made() == 3
        capture[0] = 7
        layer(x, r)  # what eager calls made is everyone's
        assert made() == 3


def test_what_a_graph_reads_is_kept_for_it(ops, capture):  # noqa: F811
    layer, x, r = make()
    with torch.no_grad():
        layer(x, r)
        old = layer.w8
        capture[0] = 1
        layer(x, r), layer(x, r)
        capture[0] = 0
        layer.requantise()
        assert [c[0][0] is old for c in layer._captured] == [True]
        assert not copy.deepcopy(layer)._captured
        for kept in layer._captured:
            kept[1].gone = lambda: True
        layer.requantise()
        assert not layer._captured


def test_a_captured_backward_pass_beside_a_living_graph_is_refused(ops, capture, monkeypatch):  # noqa: F811
    """Where it makes the parameters' gradients and the other graph is the default stream's."""
    layer, x, r = make()
    stream = [0]
    monkeypatch.setattr(layer8, "stream_of", lambda x: stream[0])
    alive = layer(x, r)
    stream[0] = capture[0] = 1
    y, _ = layer(x, r)
    before = len(ops.calls)
    for inputs in (None, [layer.weight], [x, layer.norm_weight]):
        with pytest.raises(RuntimeError, match="alive"):
            y.float().sum().backward(retain_graph=True, inputs=inputs)
    with pytest.raises(RuntimeError, match="alive"):
        torch.autograd.grad(y.float().sum(), [layer.weight], retain_graph=True)
    assert len(ops.calls) == before and layer.weight.grad is None
    xx = x * 1.0
    torch.autograd.grad(layer(xx, r.detach())[0].float().sum(), [xx])  # reaches no parameter
    capture[0] = 0
    y.float().sum().backward(retain_graph=True)  # not captured
    del alive
    capture[0] = 1
    y.float().sum().backward(retain_graph=True)
    stream[0] = 2  # made on 1, captured on 2
    layer(x, r)[0].float().sum().backward()
    for _ in range(200):
        layer(x, r)
    assert len(layer._graphs) <= 32  # those that are gone, too, but not all of them
    many = [layer(x, r) for _ in range(100)]
    assert 100 <= len(layer._graphs) <= 200 and len(many) == 100


def test_saved_before_there_were_graphs_and_captures(ops):  # noqa: F811
    """A layer or block that was pickled whole, with the attributes that it had then."""
    from paper_1611_08035_b200 import ffn8
    layer, x, r = make()
    want = layer(x, r)[0]
    state = layer.__getstate__()
    for gone in ("_captured", "_graphs"):
        del state[gone]
    old = layer8.NormLinear8.__new__(layer8.NormLinear8)
    old.__setstate__(state | {"_quantised": (layer.weight, layer.weight._version)})
    assert torch.equal(old(x, r)[0], want)
    block = ffn8.FeedForward8(256, 128, device="cpu")
    old = ffn8.FeedForward8.__new__(ffn8.FeedForward8)
    old.__setstate__(block.__getstate__() | {"_quantised": {}, "_captured": [], "_graphs": []})
    assert hasattr(old._graphs, "refuse")
