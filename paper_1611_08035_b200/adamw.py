"""AdamW on the library's step over many tensors at once (b2_adamw), with moments in 8 or in 32 bits.

In 8 bits a parameter's state takes 2 bytes and two scales for 128 elements instead of 8 bytes an element: the first moment and the root of the second one
as e4m3 numbers, rounded at random by a hash of the element's number, the step's and ``seed`` (so that steps are the same on every run).
"""
from __future__ import annotations

import torch

from . import binding as b2
from .capture import capturing
from .layer8 import _device_of

F8, E8 = torch.float8_e4m3fn, torch.float8_e8m0fnu
STATES = ("m", "v", "sm", "sv")


class AdamW(torch.optim.Optimizer):
    """``torch.optim.AdamW``'s update for float32 and bfloat16 parameters on CUDA devices.

    state_bits  8 or 32; tensors of fewer than ``least_8bit`` elements keep 32.
    capturable  keeps the learning rate and the number of the step on the device, where a captured graph of ``step()`` follows them: change ``group["lr"]`` by ``fill_``.  A number
                is shared by the parameters whose first step was the same (or who had the same number when ``group["capturable"]`` was set), and counts every step that one of them
                makes.  A captured step comes after one that was not captured, for every parameter; others are refused, as is one of a group that is not capturable.
    """

    def __init__(self, params, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=1e-2, state_bits=8, least_8bit=4096, capturable=False, seed=0):
        if state_bits not in (8, 32):
            raise ValueError(f"state_bits is {state_bits}; states have 8 or 32")
        if not all(0.0 <= b < 1.0 for b in betas) or eps < 0.0:
            raise ValueError(f"betas are {betas}, eps is {eps}: both betas lie in [0, 1), eps is not negative")
        super().__init__(params, {"lr": lr, "betas": betas, "eps": eps, "weight_decay": weight_decay, "state_bits": state_bits, "least_8bit": least_8bit, "capturable": capturable,
                                  "seed": seed})

    def add_param_group(self, group) -> None:
        super().add_param_group(group)
        for p in self.param_groups[-1]["params"]:
            if p.dtype not in (torch.float32, torch.bfloat16) or not p.is_contiguous():
                del self.param_groups[-1]
                raise ValueError(f"a parameter is {p.dtype}, {'' if p.is_contiguous() else 'not '}contiguous; the step takes contiguous float32 and bfloat16 ones")

    @staticmethod
    def _new_state(p, group) -> dict:
        n = p.numel()
        if group["state_bits"] == 32 or n < group["least_8bit"]:
            return {"step": 0, "m": torch.zeros_like(p, dtype=torch.float32), "v": torch.zeros_like(p, dtype=torch.float32)}
        zeros = lambda: torch.zeros(n, dtype=torch.uint8, device=p.device).view(F8)  # noqa: E731
        ones = lambda: torch.full(((n + 127) // 128,), 127, dtype=torch.uint8, device=p.device).view(E8)  # noqa: E731
        return {"step": 0, "m": zeros(), "v": zeros(), "sm": ones(), "sv": ones()}

    @staticmethod
    def _device_lr(group, device) -> torch.Tensor:
        lr = group["lr"]
        if not isinstance(lr, torch.Tensor) or lr.device.type != device.type:
            lr = group["lr"] = torch.tensor(float(lr), dtype=torch.float32, device=device)
        return lr if lr.device == device else lr.to(device)

    def _place_numbers(self, group, params) -> None:
        """The numbers of the steps that were made, where the group has them: in a capturable one tensors of the device, which those share who come there together with
        the same number."""
        shared: dict = {}
        for p in params:
            step = self.state[p]["step"]
            if group["capturable"] and not isinstance(step, torch.Tensor):
                if (p.device, step) not in shared:
                    shared[p.device, step] = torch.full((1,), step, dtype=torch.int64, device=p.device)
                self.state[p]["step"] = shared[p.device, step]
            elif not group["capturable"] and isinstance(step, torch.Tensor):
                if id(step) not in shared:
                    shared[id(step)] = int(step)
                self.state[p]["step"] = shared[id(step)]

    @torch.no_grad()
    def step(self, closure=None, grad_scale: torch.Tensor | None = None):
        """One step; ``grad_scale``, one float32 on the device, multiplies every gradient (clipping, loss scaling)."""
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        with_grads = [[p for p in group["params"] if p.grad is not None] for group in self.param_groups]
        for group, params in zip(self.param_groups, with_grads):  # what is refused is refused before anything is counted
            for p in params:
                if p.grad.is_sparse:
                    raise RuntimeError("AdamW does not take sparse gradients")
                st = self.state.get(p, {})  # nothing is made of a step that is refused
                if any(st[k].device != p.device for k in STATES if k in st):
                    raise RuntimeError(f"a parameter is on {p.device}, its states are not: load them again after it was moved")
                if capturing(p) and not (group["capturable"] and isinstance(st.get("step"), torch.Tensor) and isinstance(group["lr"], torch.Tensor)
                                         and group["lr"].device.type == p.device.type):
                    raise RuntimeError("a captured step is a capturable=True group's that has made one before, without the capture: its states' first values and its numbers would be a replay's")
        for number, (group, params) in enumerate(zip(self.param_groups, with_grads)):
            for p in params:
                if not self.state[p]:
                    self.state[p].update(self._new_state(p, group))
            self._place_numbers(group, params)
            calls: dict = {}  # tensors of one device and one step go together
            for p in params:
                st = self.state[p]
                step = st["step"]
                lists, _ = calls.setdefault((p.device, id(step) if group["capturable"] else step), ([[] for _ in range(6)], step))
                for to, x in zip(lists, (p, p.grad.contiguous(), *(st.get(k) for k in STATES))):
                    to.append(x)
            for (device, _), (lists, step) in calls.items():
                lr = self._device_lr(group, device) if group["capturable"] else group["lr"]
                lr = lr.to(device) if isinstance(lr, torch.Tensor) and lr.device.type == device.type else float(lr)
                with _device_of(lists[0][0]):
                    step += 1
                    try:
                        b2.b2_adamw(*lists, lr, *group["betas"], group["eps"], group["weight_decay"], step, group["seed"] + (number << 32), None if grad_scale is None else grad_scale.to(device))
                    except Exception:
                        step -= 1  # on the device, where it is the parameters' own
                        raise
                if not group["capturable"]:
                    for p in lists[0]:
                        self.state[p]["step"] = step
                torch.autograd.graph.increment_version(lists[0])  # what is made of the parameters (8-bit copies) is made anew
        return loss

    def state_dict(self) -> dict:
        """With plain numbers of steps, wherever they are counted."""
        d = super().state_dict()
        known: dict = {}
        d["state"] = {i: dict(st) for i, st in d["state"].items()}
        for st in d["state"].values():
            step = st.get("step")
            if isinstance(step, torch.Tensor):
                st["step"] = known[id(step)] if id(step) in known else known.setdefault(id(step), int(step))
        return d

    def load_state_dict(self, state_dict) -> None:
        """States and numbers of steps go to the parameters' devices, whatever device they were saved from or loaded to.  A graph that was captured before follows the old ones: capture
        again."""
        super().load_state_dict(state_dict)  # makes every floating state the parameter's type: the saved ones take their places again
        saved = state_dict["state"]
        for g, old in zip(self.param_groups, state_dict["param_groups"]):
            of_group = g.pop("step_device", None)  # where capturable groups once counted, for every parameter
            for i, p in zip(old["params"], g["params"]):
                if saved.get(i):
                    self.state[p].update({k: saved[i][k].to(p.device, copy=True) for k in STATES if k in saved[i]})
                    self.state[p]["step"] = max(map(int, of_group.values())) if of_group else int(saved[i].get("step", 0))
                    if isinstance(g["lr"], torch.Tensor) and g["capturable"]:
                        g["lr"] = g["lr"].to(p.device)
