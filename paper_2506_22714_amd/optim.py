"""AdamW over the library's kernels: all tensors of a parameter group in one launch (for every 32 of a type), states in 32 bits or in 8."""
from __future__ import annotations

import torch

from . import binding as lb


class AdamW(torch.optim.Optimizer):
    """Adam with decoupled weight decay.

    ``state_bits``: 32, or 8 for m and sqrt(v) as float8_e4m3fn with a power of two for every 256 elements, rounded by chance (``seed``).
    ``master``: 16-bit parameters are the roundings of copies in 32 bits that are kept with the states; without it every step rounds the
    parameter itself, and steps below half of its last place are lost.
    ``capturable``: the step number is kept on the GPU, so that a captured step counts on, one number for a group (a parameter without a
    gradient skips the step, the number does not); ``lr`` may then be a one-element float32 tensor there, too.  Other steps are not captured.
    Parameters are contiguous tensors of float16, bfloat16 or float32 on one GPU; gradients are of the same type."""

    def __init__(self, params, lr=1e-3, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay: float = 1e-2, state_bits: int = 32,
                 master: bool = False, capturable: bool = False, seed: int = 0):
        if state_bits not in (8, 32):
            raise ValueError(f"state_bits: {state_bits}, expected 8 or 32")
        if isinstance(lr, torch.Tensor) and not capturable:
            raise ValueError("lr: a tensor needs capturable=True")
        if not all(0 <= b < 1 for b in betas) or eps < 0:
            raise ValueError(f"betas {betas}, eps {eps}: expected betas in [0, 1) and eps >= 0")
        super().__init__(params, dict(lr=lr, betas=betas, eps=eps, weight_decay=weight_decay, state_bits=state_bits, master=master,
                                      capturable=capturable, seed=seed))

    def _new_state(self, p, group):
        if not p.is_contiguous():
            raise ValueError(f"a parameter of shape {tuple(p.shape)} is not contiguous")
        s = {} if group["capturable"] else {"step": 0}
        if group["state_bits"] == 8:
            for name in ("first", "second"):
                s[name] = torch.zeros(p.shape, dtype=torch.uint8, device=p.device).view(torch.float8_e4m3fn)
                s[name + "_scales"] = torch.ones(-(-p.numel() // lb.ADAMW_BLOCK), dtype=torch.float32, device=p.device)
        else:
            s["first"], s["second"] = (torch.zeros(p.shape, dtype=torch.float32, device=p.device) for _ in range(2))
        if group["master"] and p.dtype != torch.float32:
            s["master"] = p.detach().float()
        return s

    @staticmethod
    def _not_captured():
        if torch.cuda.is_current_stream_capturing():        # every replay would begin with new states
            raise RuntimeError("the first step makes the states: run one before the capture")

    @torch.no_grad()
    def step(self, closure=None):
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        number, runs, new = 0, [], []
        try:
            for group in self.param_groups:
                # parameters whose gradients came and went may stand at different steps: one call for each of them.  The tensor's number, by
                # which 8-bit states draw their chances, is its place among all parameters, whoever has a gradient
                calls = {}
                if not group["params"]:
                    continue
                if group["capturable"] and "step" not in group:
                    self._not_captured()
                    group["step"] = torch.zeros((), dtype=torch.int64, device=group["params"][0].device)
                for p in group["params"]:
                    number += 1
                    if p.grad is None:
                        continue
                    if p not in self.state or not self.state[p]:
                        self._not_captured()
                        self.state[p] = self._new_state(p, group)
                        new.append(p)
                    s = self.state[p]
                    calls.setdefault((p.get_device(), s.get("step")), []).append((number - 1, p, s))
                if calls and not group["capturable"] and torch.cuda.is_current_stream_capturing():      # every replay would repeat one step number
                    raise RuntimeError("a captured step needs capturable=True")
                runs.append((group, [(members, self._checked(group, members, group["step"] if step is None else step + 1))
                                     for (_, step), members in calls.items()]))
        except Exception:               # nothing has been counted or changed
            for p in new:
                del self.state[p]
            raise
        for group, calls in runs:
            if group["capturable"]:
                group["step"] += 1      # before the kernel reads it
            try:
                for members, call in calls:
                    lb._adamw_run(call)
                    for _, _, s in members:
                        if "step" in s:
                            s["step"] += 1
            except Exception:
                if group["capturable"]:
                    group["step"] -= 1
                raise
        return loss

    @torch.no_grad()
    def load_state_dict(self, state_dict):
        """The numbers of a checkpoint, wherever it was loaded to.  A rate that is a tensor stays the one that the program fills; a captured
        step has to be captured again (states are new tensors)."""
        rates = [g["lr"] for g in self.param_groups]
        super().load_state_dict(state_dict)
        # the base class converts states to their parameters' types: these keep their own
        saved = [k for g in state_dict["param_groups"] for k in g["params"]]
        for k, p in zip(saved, (p for g in self.param_groups for p in g["params"])):
            for name, x in state_dict["state"].get(k, {}).items():
                if isinstance(x, torch.Tensor):
                    self.state[p][name] = x.detach().to(p.device, copy=True)
        filled = {}                     # groups may share a rate, as long as what is loaded is the same
        for g, rate in zip(self.param_groups, rates):
            device = g["params"][0].device if g["params"] else "cpu"
            if isinstance(g.get("step"), torch.Tensor):
                g["step"] = g["step"].to(device)
            if isinstance(g["lr"], torch.Tensor):
                if isinstance(rate, torch.Tensor) and float(filled.setdefault(id(rate), g["lr"])) == float(g["lr"]):
                    g["lr"] = rate.copy_(g["lr"].reshape(rate.shape))
                else:
                    g["lr"] = g["lr"].to(device)

    def _checked(self, group, members, step):
        """The call, looked at: its tensors here, its options by a call without tensors."""
        bits8 = group["state_bits"] == 8
        params = [p for _, p, _ in members]
        states = [s for _, _, s in members]
        call = lb._adamw_checked(params, [p.grad if p.grad.is_contiguous() else p.grad.contiguous() for p in params], [s["first"] for s in states],
                                 [s["second"] for s in states], step, group["lr"], group["betas"], group["eps"], group["weight_decay"],
                                 [s["first_scales"] for s in states] if bits8 else None, [s["second_scales"] for s in states] if bits8 else None,
                                 [s.get("master") for s in states] if group["master"] else None, group["seed"], [k for k, _, _ in members])
        lb.libra_adamw(None, 0, call.opts)
        return call
