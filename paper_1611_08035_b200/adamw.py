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
    capturable  keeps the learning rate and the number of the step (a group's, not a parameter's) on the device, where a captured graph of ``step()`` follows them: change
                ``group["lr"]`` by ``fill_``.  Every parameter's first step is made before the capture; one in it is refused, as is a captured step of a group that is not capturable.
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

    def _device_numbers(self, group, device):
        """The group's learning rate and step on a device."""
        if not isinstance(group["lr"], torch.Tensor):
            group["lr"] = torch.tensor(float(group["lr"]), dtype=torch.float32, device=device)
        steps = group.setdefault("step_device", {})
        if device not in steps:
            steps[device] = torch.zeros(1, dtype=torch.int64, device=device)
        return (group["lr"] if group["lr"].device == device else group["lr"].to(device)), steps[device]

    @torch.no_grad()
    def step(self, closure=None, grad_scale: torch.Tensor | None = None):
        """One step; ``grad_scale``, one float32 on the device, multiplies every gradient (clipping, loss scaling)."""
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        for number, group in enumerate(self.param_groups):
            calls: dict = {}  # tensors of one device and one step go together
            for p in group["params"]:
                if p.grad is None:
                    continue
                if p.grad.is_sparse:
                    raise RuntimeError("AdamW does not take sparse gradients")
                st = self.state[p]
                if (not st or not group["capturable"]) and capturing(p):
                    raise RuntimeError("a captured step has capturable=True and was made once before, without the capture: its states' first values and its number would be a replay's")
                if not st:
                    st.update(self._new_state(p, group))
                st["step"] += 1
                lists = calls.setdefault((p.device, 0 if group["capturable"] else st["step"]), [[] for _ in range(6)])
                for to, x in zip(lists, (p, p.grad.contiguous(), *(st.get(k) for k in STATES))):
                    to.append(x)
            for (device, step), lists in calls.items():
                lr = group["lr"]
                if group["capturable"]:
                    lr, step = self._device_numbers(group, device)
                    step += 1
                with _device_of(lists[0][0]):
                    b2.b2_adamw(*lists, lr.to(device) if isinstance(lr, torch.Tensor) and lr.is_cuda else float(lr), *group["betas"], group["eps"], group["weight_decay"], step,
                                group["seed"] + (number << 32), None if grad_scale is None else grad_scale.to(device))
                torch.autograd.graph.increment_version(lists[0])  # what is made of the parameters (8-bit copies) is made anew
        return loss

    def load_state_dict(self, state_dict) -> None:
        super().load_state_dict(state_dict)  # makes every floating state the parameter's type: the saved ones take their places again
        saved = state_dict["state"]
        names = [i for g in state_dict["param_groups"] for i in g["params"]]
        for i, p in zip(names, (p for g in self.param_groups for p in g["params"])):
            if i in saved:
                self.state[p].update({k: saved[i][k].to(p.device, copy=True) for k in STATES if k in saved[i]})
