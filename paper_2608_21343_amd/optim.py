"""AdamW over a model's tensors in few launches (tb_adamw_step), as a torch
optimizer, with moments in 32 or in 8 bits.

Marshalling only: buffers come from torch, the step runs in libtbias.so.
"""

from __future__ import annotations

import torch

from . import capi


class AdamW(torch.optim.Optimizer):
    """AdamW (weight_decay 0: Adam) over contiguous float32 or bfloat16 parameters.

    ``state_bits`` 8 keeps a moment in one byte and a shared unit per 256 values,
    rounded so that means are kept (the roundings follow from ``seed``).
    ``master`` keeps a float32 copy of bfloat16 parameters, which the steps
    update. ``capturable``: the number of the step lives on the device, so that a
    captured graph of ``step`` can be replayed as a training loop, once a first
    step has made the states; every parameter then needs a gradient in every step,
    and a learning rate that changes is a device tensor of one float32.
    ``step(grad_scale=...)`` takes a device tensor of one float32 that multiplies the
    gradients, as clipping needs it."""

    def __init__(self, params, lr=1e-3, betas=(0.9, 0.999), eps: float = 1e-8,
                 weight_decay: float = 0.01, state_bits: int = 32, master: bool = False,
                 capturable: bool = False, seed: int = 0):
        super().__init__(params, dict(lr=lr, betas=betas, eps=eps, weight_decay=weight_decay,
                                      state_bits=state_bits, master=master,
                                      capturable=capturable, seed=seed))

    def add_param_group(self, group):
        super().add_param_group(group)
        try:
            self._check(self.param_groups[-1])
        except ValueError:
            self.param_groups.pop()  # (a group that is refused leaves nothing behind)
            raise

    @staticmethod
    def _check(group):
        if group["state_bits"] not in (8, 32):
            raise ValueError("state_bits must be 8 or 32")
        lr = group["lr"]
        if isinstance(lr, torch.Tensor) and (lr.numel() != 1 or lr.dtype != torch.float32):
            raise ValueError("a learning rate on the device is one float32")
        for p in group["params"]:
            if p.dtype not in (torch.float32, torch.bfloat16):
                raise ValueError("parameters must be float32 or bfloat16")
            if not p.is_contiguous():
                raise ValueError("parameters must be contiguous")

    def _start(self, p, group):
        s = self.state[p]
        if s:
            return s
        if torch.cuda.is_current_stream_capturing():
            # (its replays would begin with empty states every time)
            raise RuntimeError("the first step makes the states: run it before the capture")
        if group["state_bits"] == 8:
            units = (p.numel() + 255) // 256
            for name in ("exp_avg", "exp_avg_sq"):
                s[name] = torch.zeros(p.shape, dtype=torch.uint8, device=p.device)
                s[name + "_unit"] = torch.zeros(units, dtype=torch.float32, device=p.device)
        else:
            for name in ("exp_avg", "exp_avg_sq"):
                s[name] = torch.zeros(p.shape, dtype=torch.float32, device=p.device)
        if group["master"] and p.dtype == torch.bfloat16:
            s["master"] = p.detach().float()
        s["step"] = 0
        return s

    @torch.no_grad()
    def step(self, closure=None, grad_scale=None):
        if torch.cuda.is_current_stream_capturing() and not all(
                group["capturable"] for group in self.param_groups):
            # (a graph would hold this step's bias corrections and roundings)
            raise RuntimeError("a step is captured of capturable groups alone, and its states "
                               "are made before the capture")
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        for at, group in enumerate(self.param_groups):
            if "step_dev" in group and not group["capturable"]:
                self._count_on_host(group)
            # one call for the tensors of a device and type that are equally far
            calls = {}
            for p in group["params"]:
                if p.grad is None:
                    if group["capturable"]:
                        raise RuntimeError("a capturable step needs every gradient")
                    continue
                if p.grad.is_sparse:
                    raise RuntimeError("sparse gradients are not supported")
                s = self._start(p, group)
                if not group["capturable"]:
                    s["step"] += 1
                calls.setdefault((p.device, p.dtype, s["step"]), []).append((p, s))
            for (device, dtype, step), some in calls.items():
                self._call(group, at, device, step, [p for p, _ in some], [s for _, s in some],
                           grad_scale)
        return loss

    def _counter(self, group, device):
        """The number of a capturable group's steps so far, on a device."""
        counters = group.setdefault("step_dev", {})
        if device not in counters:
            if torch.cuda.is_current_stream_capturing():
                # (its replays would count from the same number every time)
                raise RuntimeError("the first capturable step makes its counter: run it before "
                                   "the capture")
            steps = {self.state[p]["step"] for p in group["params"]}
            if len(steps) != 1:
                raise RuntimeError("parameters that have made different numbers of steps cannot "
                                   "become capturable")
            counters[device] = torch.full((1,), steps.pop(), dtype=torch.int64, device=device)
        return counters[device]

    def _count_on_host(self, group):
        """Of a group that was capturable: its states take over the number of its steps."""
        counters = group.pop("step_dev")
        for p in group["params"]:
            if p in self.state and p.device in counters:
                self.state[p]["step"] = int(counters[p.device])

    def _call(self, group, at, device, step, params, states, grad_scale):
        lr, lr_dev, step_dev = group["lr"], None, None
        if isinstance(lr, torch.Tensor):
            lr, lr_dev = 0.0, lr.reshape(1)
        if group["capturable"]:
            # (the tensors of a device share it: the first call of a step counts)
            step_dev = self._counter(group, device)
            if params[0] is next(p for p in group["params"] if p.device == device):
                step_dev.add_(1)
            step = 1
        more = {}
        if group["state_bits"] == 8:
            more = dict(m_unit=[s["exp_avg_unit"] for s in states],
                        v_unit=[s["exp_avg_sq_unit"] for s in states],
                        seed=group["seed"] + 0x9e3779b9 * at)
        if "master" in states[0]:
            more["master"] = [s["master"] for s in states]
        capi.tb_adamw_step(params, [p.grad.contiguous() for p in params],
                           [s["exp_avg"] for s in states], [s["exp_avg_sq"] for s in states],
                           lr=lr, beta1=group["betas"][0], beta2=group["betas"][1],
                           eps=group["eps"], weight_decay=group["weight_decay"], step=step,
                           lr_dev=lr_dev, step_dev=step_dev, grad_scale=grad_scale, **more)
        # the library writes by address: graphs that still need these notice
        for p in params:
            torch.autograd.graph.increment_version(p)

    def load_state_dict(self, state_dict):
        super().load_state_dict(state_dict)
        # counters and rates on the device were saved with their group, under the devices of then
        for group in self.param_groups:
            devices = {p.device for p in group["params"]}
            counters = group.pop("step_dev", None)
            if counters:
                steps = max(int(t) for t in counters.values())  # (they are the same on all)
                group["step_dev"] = {d: torch.full((1,), steps, dtype=torch.int64, device=d)
                                     for d in devices}
            if isinstance(group["lr"], torch.Tensor) and len(devices) == 1:
                group["lr"] = group["lr"].to(*devices)
        # the states keep their own types (torch casts them to the parameter's)
        saved = [i for g in state_dict["param_groups"] for i in g["params"]]
        mine = [p for g in self.param_groups for p in g["params"]]
        for i, p in zip(saved, mine):
            for name, value in state_dict["state"].get(i, {}).items():
                if isinstance(value, torch.Tensor):
                    self.state[p][name] = value.detach().clone().to(p.device)
