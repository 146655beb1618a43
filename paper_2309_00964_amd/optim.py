"""AdamW for clustered training: dL/dw of the clustering's backward to the next
step's weights.

``AdamW`` is a ``torch.optim.Optimizer`` whose step is the library's
``adamw_batch``: many tensors per launch, moments in fp32 or in 8 bits (float8
with one fp32 scale per 256 elements, see include/edkm.h), and optionally fp32
master copies of 16-bit weights, whose updates would else be lost below half a
step.  Argument marshalling only: every step runs in the HIP library.
"""
from __future__ import annotations

import torch

from . import edkm

_PARAM_TYPES = (torch.float16, torch.bfloat16, torch.float32)


def _check_group(group):
    """Refuses options, the defaults' or a group's own, and parameters that a step cannot take."""
    lr, betas = group["lr"], group["betas"]
    if group["state_bits"] not in (8, 32):
        raise ValueError("state_bits must be 8 or 32")
    if isinstance(lr, torch.Tensor):
        if lr.numel() != 1 or lr.dtype != torch.float32:
            raise ValueError("a tensor lr must be one float32")
    elif not 0 <= lr < float("inf"):
        raise ValueError("lr must be finite and not negative")
    if not (0 <= betas[0] < 1 and 0 <= betas[1] < 1):
        raise ValueError("betas must be in [0, 1)")
    if not 0 <= group["eps"] < float("inf") or not 0 <= group["weight_decay"] < float("inf"):
        raise ValueError("eps and weight_decay must be finite and not negative")
    for p in group["params"]:
        if p.dtype not in _PARAM_TYPES:
            raise ValueError("parameters must be fp16, bf16 or float32, not %s" % p.dtype)


class AdamW(torch.optim.Optimizer):
    """AdamW with decoupled weight decay over fp16, bf16 and float32 parameters on a GPU.

    lr: a number, or a one-element float32 tensor on the parameters' device (a
    captured step then follows it); state_bits: 32 or 8; master_weights: keep
    fp32 copies of 16-bit parameters; seed: of the 8-bit states' rounding noise.

    The number of steps done lives on the device (one counter for the parameters
    that have taken the same steps), so a step can be captured in a HIP graph,
    once a first step outside has made the states.  A step leaves parameters
    without gradient alone.
    """

    def __init__(self, params, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, state_bits=32,
                 master_weights=False, seed=0):
        super().__init__(params, dict(lr=lr, betas=tuple(betas), eps=eps, weight_decay=weight_decay, state_bits=state_bits,
                                      master_weights=bool(master_weights), seed=int(seed)))

    def add_param_group(self, group):
        super().add_param_group(group)
        try:
            _check_group(self.param_groups[-1])
        except Exception:
            del self.param_groups[-1]
            raise

    def _new_state(self, p, group, step):
        if not p.is_cuda or not p.is_contiguous():
            raise ValueError("parameters must be contiguous GPU tensors")
        n, dev = p.numel(), p.device
        s = self.state[p]
        s["step"] = step
        if group["state_bits"] == 8:
            blocks = (n + edkm.STATE_BLOCK - 1) // edkm.STATE_BLOCK
            s["exp_avg"] = torch.zeros(n, dtype=torch.uint8, device=dev).view(torch.float8_e4m3fn)
            s["exp_avg_sq"] = torch.zeros(n, dtype=torch.uint8, device=dev).view(torch.float8_e5m2)
            s["exp_avg_scale"] = torch.zeros(blocks, dtype=torch.float32, device=dev)
            s["exp_avg_sq_scale"] = torch.zeros(blocks, dtype=torch.float32, device=dev)
        else:
            s["exp_avg"] = torch.zeros(n, dtype=torch.float32, device=dev)
            s["exp_avg_sq"] = torch.zeros(n, dtype=torch.float32, device=dev)
        if group["master_weights"] and p.dtype != torch.float32:
            s["master"] = p.detach().float().reshape(-1)

    def _counters(self, active):
        """A state for every active parameter, and a counter of its own for the active part
        of a cohort (the parameters that share a counter) whose other part sits this step out."""
        capturing = any(p.is_cuda for _, p in active[:1]) and torch.cuda.is_current_stream_capturing()
        fresh, cohorts = {}, {}
        for group in self.param_groups:
            for p in group["params"]:
                s = self.state.get(p)
                if s:
                    cohorts.setdefault(id(s["step"]), [s["step"], 0, []])[1] += 1
        for group, p in active:
            if not self.state.get(p):
                if capturing:
                    raise RuntimeError("take a first step outside the capture: it makes the states")
                step = fresh.get(p.device)
                if step is None:
                    step = fresh[p.device] = torch.zeros(1, dtype=torch.int32, device=p.device)
                self._new_state(p, group, step)
            elif id(self.state[p]["step"]) in cohorts:
                cohorts[id(self.state[p]["step"])][2].append(p)
        for step, members, present in cohorts.values():
            if present and len(present) < members:
                if capturing:
                    raise RuntimeError("parameters that took the same steps so far do not all have a gradient; "
                                       "take such a step outside the capture first")
                own = step.clone()
                for p in present:
                    self.state[p]["step"] = own

    @torch.no_grad()
    def step(self, closure=None):
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        active = [(group, p) for group in self.param_groups for p in group["params"] if p.grad is not None]
        for _, p in active:
            if p.grad.is_sparse:
                raise RuntimeError("sparse gradients are not supported")
            if p.grad.dtype != p.dtype and p.grad.dtype != torch.float32:
                raise RuntimeError("a gradient must have its parameter's type or float32")
        self._counters(active)
        # one call per counter, hyperparameters and types; the counter advances once a step,
        # with the last call on it
        calls = {}
        for g, group in enumerate(self.param_groups):
            for p in group["params"]:
                if p.grad is not None:
                    s = self.state[p]
                    key = (g, id(s["step"]), p.device, p.dtype, p.grad.dtype, "master" in s)
                    calls.setdefault(key, []).append(p)
        users = {}
        for key in calls:
            users.setdefault(key[1], []).append(key)
        for key, ps in calls.items():
            group, ss = self.param_groups[key[0]], [self.state[p] for p in ps]
            last = users[key[1]][-1] == key
            step = ss[0]["step"]
            eight = group["state_bits"] == 8
            edkm.adamw_batch([p.detach().view(-1) for p in ps], [p.grad.contiguous().view(-1) for p in ps],
                             [s["exp_avg"] for s in ss], [s["exp_avg_sq"] for s in ss], step if last else step.clone(),
                             group["lr"], group["betas"][0], group["betas"][1], group["eps"], group["weight_decay"],
                             masters=[s["master"] for s in ss] if key[5] else None,
                             m_scales=[s["exp_avg_scale"] for s in ss] if eight else None,
                             v_scales=[s["exp_avg_sq_scale"] for s in ss] if eight else None, seed=group["seed"])
            # the library writes through pointers: autograd's check of saved tensors hears of it here
            torch.autograd.graph.increment_version(ps)
        return loss

    def load_state_dict(self, state_dict):
        """torch's, but with every state tensor in its own type (torch casts them to the
        parameter's), the counters shared as they were saved, and rates that are tensors on
        their parameters' device."""
        super().load_state_dict(state_dict)
        rates = {}
        for group in self.param_groups:
            if isinstance(group["lr"], torch.Tensor) and group["params"]:
                lr, device = group["lr"], group["params"][0].device
                group["lr"] = rates.setdefault((id(lr), device), lr.to(device))
        saved = state_dict["state"]
        ids = [i for group in state_dict["param_groups"] for i in group["params"]]
        params = [p for group in self.param_groups for p in group["params"]]
        steps = {}
        for i, p in zip(ids, params):
            if i not in saved:
                continue
            for name, value in saved[i].items():
                if name == "step":
                    key = (id(value), p.device)
                    if key not in steps:
                        steps[key] = value.detach().to(p.device, copy=True)
                    self.state[p][name] = steps[key]
                else:
                    self.state[p][name] = value.detach().to(p.device, copy=True)
