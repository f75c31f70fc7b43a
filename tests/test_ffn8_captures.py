"""The feed-forward block in several captures, without a GPU: captures are told apart by their numbers, the operators are test_ffn8.py's stand-in."""
import pytest
import torch

from paper_1611_08035_b200 import binding, ffn8
from test_ffn8 import make, ops  # noqa: F401


@pytest.fixture
def capture(monkeypatch):
    """The number of the capture that calls go into; 0: none."""
    now = [0]
    monkeypatch.setattr(ffn8, "capturing", lambda x: now[0] != 0)
    monkeypatch.setattr(ffn8, "capture_id", lambda x: now[0])
    return now


def test_what_one_capture_made_is_not_another_ones(ops, capture):  # noqa: F811
    block, x, r = make()
    with torch.no_grad():
        capture[0] = 5
        block(x, r), block(x, r)
        assert ops.calls.count("quant") == 2
        capture[0] = 6  # whose graph may run before the other's
        block(x, r), block(x, r)
        assert ops.calls.count("quant") == 4
        capture[0] = 0
        block(x, r)
        assert ops.calls.count("quant") == 6
        capture[0] = 7
        block(x, r)  # what eager calls made is everyone's
        assert ops.calls.count("quant") == 6


def test_a_refused_capture_leaves_nothing_behind(ops, capture):  # noqa: F811
    block, x, r = make()
    y = block(x, r)
    block._graphs[0] = (block._graphs[0][0], 7)  # as if from another stream
    with torch.no_grad():
        block.up.mul_(2.0)
    before, kept = ops.calls.count("quant"), len(block._captured)
    capture[0] = 1
    with pytest.raises(RuntimeError, match="alive"):
        block(x, r)
    assert ops.calls.count("quant") == before and len(block._captured) == kept
    del y
    capture[0] = 2
    block(x, r)
    assert ops.calls.count("quant") == before + 2


def test_the_number_of_a_capture_has_to_have_a_place(b2):
    assert b2.lib().b2_graph_capture_id(None, None) == -2
    assert "b2_graph_capture_id" in binding.EXPORTED_SYMBOLS


def test_no_event_is_refused(b2):
    assert b2.lib().b2_event_finish(None) == -1


def test_kept_once_for_each_capture(ops, capture):  # noqa: F811
    block, x, r = make()
    with torch.no_grad():
        block(x, r)
        capture[0] = 1
        for _ in range(3):
            block(x, r)
        assert len(block._captured) == 1
        capture[0] = 2
        block(x, r)
        assert len(block._captured) == 2  # the other graph may go first
        block.requantise()
        block(x, r)  # made in the capture: its graph's own
        assert len(block._captured) == 2
        for kept in block._captured:
            kept[2].gone = lambda: True
        block.requantise()
        assert not block._captured


def test_what_is_no_watch_is_refused(b2):
    for watch in (-1, 0, 4096):
        assert b2.lib().b2_graph_gone(watch) == 0 and b2.lib().b2_graph_unwatch(watch) == -1
    assert b2.lib().b2_graph_watch(None, None) == -2


def test_a_captured_backward_pass_beside_a_living_graph(ops, capture, monkeypatch):  # noqa: F811
    """Beside a graph whose backward pass has run, calls are captured; a backward pass is refused where it makes the parameters' gradients and the graph is the default stream's."""
    block, x, r = make()
    stream = [0]
    monkeypatch.setattr(ffn8, "stream_of", lambda x: stream[0])
    alive = block(x, r)
    alive.float().sum().backward(retain_graph=True)
    block.zero_grad()
    stream[0] = capture[0] = 1
    y = block(x, r)
    before = len(ops.calls)
    with pytest.raises(RuntimeError, match="alive"):
        y.float().sum().backward(retain_graph=True)
    with pytest.raises(RuntimeError, match="alive"):
        torch.autograd.grad(y.float().sum(), [block.down], retain_graph=True)
    assert len(ops.calls) == before and block.down.grad is None
    del alive
    y.float().sum().backward(retain_graph=True)
    stream[0] = 2  # made and run on 1, captured on 2
    block(x, r).float().sum().backward()
