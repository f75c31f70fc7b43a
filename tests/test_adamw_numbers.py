"""The numbers of steps that the optimiser hands over, without a GPU: a stand-in takes the calls."""
import pytest
import torch

from paper_1611_08035_b200 import adamw


@pytest.fixture
def calls(monkeypatch):
    """(parameters, number of the step) of every call."""
    taken = []

    class Take:
        @staticmethod
        def b2_adamw(p, g, m, v, sm, sv, lr, b1, b2, eps, wd, step, seed, scale):
            taken.append((len(p), int(step)))

    monkeypatch.setattr(adamw, "b2", Take)
    return taken


def make(n=2, **kw):
    params = [torch.nn.Parameter(torch.zeros(5000)) for _ in range(n)]
    return params, adamw.AdamW(params, **kw)


def go(opt, params, steps=1):
    for p in params:
        p.grad = torch.ones(5000)
    for _ in range(steps):
        opt.step()
    opt.zero_grad()


def test_capturable_goes_on_counting(calls):
    """Set after steps were made, as where a training that was resumed is captured; and taken back, after replays that nobody but the device has counted."""
    params, opt = make()
    go(opt, params, 100)
    opt.param_groups[0]["capturable"] = True
    go(opt, params, 2)
    assert calls[98:] == [(2, 99), (2, 100), (2, 101), (2, 102)]
    opt.state[params[0]]["step"] += 7  # seven replays of a captured step
    opt.param_groups[0]["capturable"] = False
    go(opt, params, 2)
    assert calls[102:] == [(2, 110), (2, 111)]


def test_numbers_are_the_parameters(calls):
    """A parameter that comes later counts from its own first step, capturable or not, and after a change."""
    for capturable in (False, True):
        calls.clear()
        (a, b), opt = make(capturable=capturable)
        go(opt, [a], 3)
        go(opt, [a, b], 2)
        assert sorted(calls[3:]) == [(1, 1), (1, 2), (1, 4), (1, 5)]
        opt.param_groups[0]["capturable"] = not capturable
        go(opt, [a, b])
        assert sorted(calls[7:]) == [(1, 3), (1, 6)]


def test_a_number_that_a_capture_would_make_is_refused(calls, monkeypatch):
    params, opt = make()
    go(opt, params, 4)
    opt.param_groups[0]["capturable"] = True
    monkeypatch.setattr(adamw, "capturing", lambda x: True)
    with pytest.raises(RuntimeError, match="capture"):
        go(opt, params)
    monkeypatch.setattr(adamw, "capturing", lambda x: False)
    go(opt, params)
    monkeypatch.setattr(adamw, "capturing", lambda x: True)
    go(opt, params)
    assert calls[4:] == [(2, 5), (2, 6)]
    opt.param_groups[0]["lr"] = 1e-4  # a number in place of the tensor that the graph would follow
    with pytest.raises(RuntimeError, match="capture"):
        go(opt, params)


@pytest.mark.parametrize("capturable", [False, True])
def test_refused_steps_do_not_count(calls, capturable, monkeypatch):
    """Neither those that the optimiser refuses nor those that the binding does."""
    (a, b), opt = make(capturable=capturable)
    go(opt, [a, b], 2)
    a.grad, b.grad = torch.ones(5000), torch.ones(5000).to_sparse()
    with pytest.raises(RuntimeError, match="sparse"):
        opt.step()
    monkeypatch.setattr(adamw, "capturing", lambda x: x is b)
    b.grad = torch.ones(5000)
    opt.state[b]["step"] = int(opt.state[b]["step"])  # not the device's
    with pytest.raises(RuntimeError, match="capture"):
        opt.step()
    monkeypatch.setattr(adamw, "capturing", lambda x: False)
    taken = adamw.b2.b2_adamw

    def refuse(*args):
        raise TypeError

    monkeypatch.setattr(adamw.b2, "b2_adamw", staticmethod(refuse))
    versions = a._version, b._version
    for _ in range(3):
        with pytest.raises(TypeError):
            opt.step()
    monkeypatch.setattr(adamw.b2, "b2_adamw", staticmethod(taken))
    assert (a._version, b._version) == versions and [int(opt.state[p]["step"]) for p in (a, b)] == [2, 2]
    calls.clear()
    go(opt, [a, b])
    assert [step for _, step in calls] == [3] * len(calls) and sum(n for n, _ in calls) == 2
