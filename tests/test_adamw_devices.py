"""Tensors of several devices in one step, without a GPU: refused before anything is launched."""
import pytest
import torch

from paper_1611_08035_b200 import adamw
from test_adamw_numbers import calls, go, make  # noqa: F401

E4M3, E8M0, F32 = torch.float8_e4m3fn, torch.float8_e8m0fnu, torch.float32


class OnDevice:
    """What the binding asks of a tensor, for one on a device that is not here."""

    is_cuda = True

    def __init__(self, n, dtype, index):
        self.n, self.dtype, self.device, self.shape = n, dtype, torch.device("cuda", index), (n,)

    def numel(self):
        return self.n

    def is_contiguous(self):
        return True

    def data_ptr(self):
        raise AssertionError("the address of a tensor of a refused call was asked for")


def test_the_binding(b2):
    full = b2._connected.get("b2_adamw", (None, b2.b2_adamw))[1]
    for other in range(6):
        where = [1 if i == other else 0 for i in range(6)]
        types = (F32, F32, E4M3, E4M3, E8M0, E8M0)
        one = [[OnDevice(256 if i < 4 else 2, t, w)] for i, (t, w) in enumerate(zip(types, where))]
        with pytest.raises(ValueError, match="one device"):
            full(*one, 1e-3, 0.9, 0.99, 1e-8, 0.0, 1)
    two = [[OnDevice(256 if i < 4 else 2, t, w) for w in (0, 1)] for i, t in enumerate(types)]
    with pytest.raises(ValueError, match="one device"):
        full(*two, 1e-3, 0.9, 0.99, 1e-8, 0.0, 1)


def test_a_parameter_that_was_moved(calls):  # noqa: F811
    params, opt = make()
    go(opt, params)
    for k in ("m", "v", "sm", "sv"):
        state = opt.state[params[1]]
        kept, state[k] = state[k], state[k].to("meta")
        with pytest.raises(RuntimeError, match="moved"):
            go(opt, params)
        state[k] = kept
    assert calls == [(2, 1)]
    go(opt, params)
    assert calls == [(2, 1), (2, 2)]
