"""AdamW on this library's step over many tensors (AsdOps.adamw), as a torch optimizer.

    opt = AdamW(net.parameters(), lr=1e-3)                    moments in float32
    opt = AdamW(net.parameters(), lr=1e-3, state_bits=8)      moments in 8 bits with two scales to 256 of them

Parameters in float16 or bfloat16 get a float32 master value, which the step changes and rounds to the parameter: products read
the 16-bit parameter as it is, with no cast of their own (masters=False: the parameter itself is changed, and rounded).  What else
writes to a parameter is taken over into its master value: where the two no longer agree the next step begins from the
parameter.  It sees that a parameter was written to by its version, which a write through .data or in a replayed graph does not
change: refresh_masters() is for those.  Moments in 8 bits are rounded up with the probability of their fraction, so that they follow
decays of less than half of their steps.
"""
from __future__ import annotations

import torch

from .operators import default_ops


class AdamW(torch.optim.Optimizer):
    """Parameters are contiguous CUDA tensors; one without a gradient is left as it is and its steps are not counted.  lr may be
    a float32 tensor of one element on the device, which a captured step then reads.  A step may be captured in a CUDA
    graph once every parameter has its state, that is after a first step; the parameters that it steps together then do so for good: a
    step in which some of them have no gradient is refused.  Parameters that take different steps are counted apart, with a launch for
    each count."""

    def __init__(self, params, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=1e-2, state_bits=32, masters=True):
        if state_bits not in (8, 32):
            raise ValueError(f"state_bits must be 8 or 32: {state_bits}")
        for name, v in (("eps", eps), ("weight_decay", weight_decay), *([] if torch.is_tensor(lr) else [("lr", lr)])):
            if not 0 <= v < float("inf"):
                raise ValueError(f"{name} must be finite and >= 0: {v}")
        if not all(0 <= b < 1 for b in betas):
            raise ValueError(f"betas must be in [0, 1): {betas}")
        self._captured = {}  # counters that a captured step moves on, by their identity
        self._versions = {}  # of parameters with a master value after their last step, by their identity
        super().__init__(params, dict(lr=lr, betas=tuple(betas), eps=eps, weight_decay=weight_decay, state_bits=state_bits, masters=masters))

    def __setstate__(self, state):
        super().__setstate__(state)
        self._captured, self._versions = {}, {}

    def _new_state(self, p, group, fresh):
        if not p.is_cuda or not p.is_contiguous():
            raise RuntimeError("AdamW: parameters must be contiguous CUDA tensors")
        if torch.cuda.is_current_stream_capturing():
            raise RuntimeError("AdamW: a parameter has no state yet: take a step before one is captured")
        if p.device not in fresh:  # those that begin together share a counter
            fresh[p.device] = torch.zeros(2, dtype=torch.int64, device=p.device)
        wide = group["state_bits"] == 32
        state = {"step": fresh[p.device], "exp_avg": torch.zeros(p.shape, dtype=torch.float32 if wide else torch.int8, device=p.device),
                 "exp_avg_sq": torch.zeros(p.shape, dtype=torch.float32 if wide else torch.uint8, device=p.device)}
        if not wide:
            state["scales"] = torch.zeros(((p.numel() + 255) // 256, 2), device=p.device)
        if group["masters"] and p.dtype != torch.float32:
            state["master"] = p.detach().float()
            self._versions[id(p)] = None if p.is_inference() else p._version
        self.state[p] = state

    def _plan(self, group):
        """The group's parameters that have a gradient by the counter of their steps, which those share that have taken the same ones, those
        without a state, and the counters that only some of those that share them move on this time.  Nothing is changed yet."""
        ready, waiting, new = {}, set(), []
        for p in group["params"]:
            if p.grad is None:
                if p in self.state:
                    waiting.add(id(self.state[p]["step"]))
                continue
            if p.grad.is_sparse:
                raise RuntimeError("AdamW: sparse gradients are not supported")
            if p in self.state:
                ready.setdefault(id(self.state[p]["step"]), []).append(p)
            else:
                new.append(p)
        split = [key for key in ready if key in waiting]
        if split and torch.cuda.is_current_stream_capturing():
            raise RuntimeError("AdamW: parameters that have stepped together so far no longer do: take such a step before one is captured")
        if any(key in self._captured for key in split):  # its replays count the steps of all of them in one place
            raise RuntimeError("AdamW: parameters whose steps were captured together cannot step apart; load_state_dict(state_dict()) parts the "
                               "optimizer from the captured step, which then has to be captured again")
        return ready, new, split

    def _calls(self, group, ready, new, split):
        """Lists of parameters that step together."""
        for key in split:
            step = self.state[ready[key][0]]["step"].clone()
            for p in ready[key]:
                self.state[p]["step"] = step
        fresh = {}
        for p in new:
            self._new_state(p, group, fresh)
            ready.setdefault(id(self.state[p]["step"]), []).append(p)
        return ready.values()

    @torch.no_grad()
    def _refresh(self, p, master):
        """The elements of a master value that are not what its parameter was rounded from; the others keep their low bits."""
        master.copy_(torch.where(p == master.to(p.dtype), master, p))

    def refresh_masters(self):
        """Takes over what parameters have been set to into their master values, however they were written."""
        for p, state in self.state.items():
            if "master" in state:
                self._refresh(p, state["master"])

    @torch.no_grad()
    def step(self, closure=None, grad_scale=None, skip=None):
        """grad_scale: a factor of the gradients; skip: nonzero for a step that is to be left out; float32 tensors of one element on
        the device, or None."""
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        plans = [(group, self._plan(group)) for group in self.param_groups]
        for group, plan in plans:
            for params in self._calls(group, *plan):
                states = [self.state[p] for p in params]
                masters = [s.get("master") for s in states]
                for p, master in zip(params, masters):
                    if master is not None and not p.is_inference() and self._versions.get(id(p)) != p._version:
                        self._refresh(p, master)
                with torch.cuda.device(params[0].device):
                    if torch.cuda.is_current_stream_capturing():
                        self._captured[id(states[0]["step"])] = states[0]["step"]
                    default_ops().adamw(params, [p.grad for p in params], [s["exp_avg"] for s in states], [s["exp_avg_sq"] for s in states],
                                        states[0]["step"], lr=group["lr"], betas=group["betas"], eps=group["eps"], weight_decay=group["weight_decay"],
                                        masters=masters,
                                        scales=[s["scales"] for s in states] if group["state_bits"] == 8 else None, grad_scale=grad_scale, skip=skip,
                                        unbiased=group["state_bits"] == 8)
                self._versions.update((id(p), p._version) for p, master in zip(params, masters) if master is not None and not p.is_inference())
        return loss

    def load_state_dict(self, state_dict):
        """As torch's, but the states keep their types (torch's would give them the parameters'), and parameters that have taken the same
        number of steps share its counter again."""
        super().load_state_dict(state_dict)
        self._captured, self._versions = {}, {}  # the states are other tensors now
        ids = [i for group in state_dict["param_groups"] for i in group["params"]]
        params = [p for group in self.param_groups for p in group["params"]]
        for i, p in zip(ids, params):
            if i in state_dict["state"]:
                self.state[p] = {k: v.detach().to(p.device, copy=True) if torch.is_tensor(v) else v for k, v in state_dict["state"][i].items()}
        for group in self.param_groups:
            counters = {}
            for p in group["params"]:
                if p in self.state:
                    step = self.state[p]["step"]
                    self.state[p]["step"] = counters.setdefault((p.device, int(step[0])), step)
