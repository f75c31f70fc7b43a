"""Saving and loading the optimiser, without a GPU: a stand-in takes the calls."""
import copy
import io

import pytest
import torch

from paper_1611_08035_b200 import adamw
from test_adamw_numbers import calls, go, make  # noqa: F401


@pytest.mark.parametrize("to", [False, True])
@pytest.mark.parametrize("capturable", [False, True])
def test_the_number_goes_on(calls, capturable, to):  # noqa: F811
    params, opt = make(capturable=capturable)
    go(opt, params[:1], 2)
    go(opt, params, 3)
    if capturable:
        opt.state[params[0]]["step"] += 4  # replays
    file = io.BytesIO()
    torch.save(opt.state_dict(), file)
    file.seek(0)
    saved = torch.load(file, map_location="cpu")
    assert all(type(st["step"]) is int for st in saved["state"].values())
    calls.clear()
    others, other = make(capturable=to)
    other.load_state_dict(saved)
    other.param_groups[0]["capturable"] = to
    go(other, others)
    first = 6 + 4 * capturable
    assert sorted(calls) == [(1, 4), (1, first)]
    go(opt, params)
    assert sorted(calls[2:]) == [(1, 4), (1, first)]  # the saved one goes on, too


def test_the_saved_state_is_no_ones(calls):  # noqa: F811
    params, opt = make(capturable=True)
    go(opt, params)
    saved = opt.state_dict()
    before = copy.deepcopy(saved)
    others, other = make()
    other.load_state_dict(saved)
    go(other, others, 3), go(opt, params, 2)
    for i in before["state"]:
        assert saved["state"][i]["step"] == before["state"][i]["step"] == 1
    assert other.state[others[0]]["step"].tolist() == [4] and opt.state[params[0]]["step"].tolist() == [3]


def test_numbers_that_a_group_kept(calls):  # noqa: F811
    """The older form of a capturable group's state: a counter for each device, and numbers of the parameters that replays did not reach."""
    params, opt = make()
    go(opt, params, 2)
    saved = opt.state_dict()
    saved["param_groups"][0] |= {"capturable": True, "step_device": {torch.device("cuda:0"): torch.tensor([40])}}
    opt.load_state_dict(saved)
    go(opt, params)
    assert calls[-1] == (2, 41) and "step_device" not in opt.param_groups[0]


def test_the_learning_rate_goes_to_the_device(calls, monkeypatch):  # noqa: F811
    """A rate that was loaded to another kind of device would be no number that a graph can follow."""
    params, opt = make(capturable=True)
    go(opt, params)
    saved = opt.state_dict()
    assert isinstance(saved["param_groups"][0]["lr"], torch.Tensor)
    saved["param_groups"][0]["lr"] = saved["param_groups"][0]["lr"].to("meta")
    moved = []
    monkeypatch.setattr(torch.Tensor, "to", (lambda to: lambda x, *a, **k: (moved.append(a), torch.zeros(()))[1] if x.device.type == "meta" else to(x, *a, **k))(torch.Tensor.to))
    opt.load_state_dict(saved)
    assert moved and opt.param_groups[0]["lr"].device.type == "cpu"


def test_a_refused_step_leaves_nothing_to_save(calls):  # noqa: F811
    params, opt = make()
    go(opt, params[:1])
    params[0].grad, params[1].grad = torch.ones(5000), torch.ones(5000).to_sparse()
    with pytest.raises(RuntimeError):
        opt.step()
    saved = opt.state_dict()
    assert list(saved["state"]) == [0]
    saved["state"][1] = {}  # as an optimiser that looked at what is not there had it
    others, other = make()
    other.load_state_dict(saved)
    go(other, others)
    assert sorted(calls[1:]) == [(1, 1), (1, 2)] and set(other.state[others[1]]) == {"step", "m", "v", "sm", "sv"}
