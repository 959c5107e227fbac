"""Torch front door to the multi-tensor AdamW step: `AdamW(params, ...)`, a torch.optim.Optimizer whose step() is one
fq_adamw_step call (one launch) per parameter group, or for each step number in it where some had their first gradient late.

Marshalling only.  The moments are float32, or float8_e4m3fn codes with a scale per 256 elements (`states="float8"`, a quarter
of the memory, rounded stochastically).  There is no CPU path: CPU parameters raise.
"""
import math
import weakref

import torch

from . import binding as fq

_DTYPES = (torch.float16, torch.float32)


def _check_rates(group):
    """What the library would refuse in a step."""
    lr, (beta1, beta2), eps, decay = group["lr"], group["betas"], group["eps"], group["weight_decay"]
    if not (math.isfinite(lr) and 0.0 <= beta1 < 1.0 and 0.0 <= beta2 < 1.0 and math.isfinite(eps) and eps >= 0.0 and math.isfinite(decay)):
        raise ValueError("lr %r, betas %r, eps %r or weight_decay %r is out of range" % (lr, (beta1, beta2), eps, decay))


def _check_group(group):
    if group["states"] not in ("float32", "float8"):
        raise ValueError("states must be float32 or float8, not %r" % (group["states"],))
    for p in group["params"]:
        if not p.is_cuda:
            raise RuntimeError("AdamW runs on the GPU only (no CPU fallback)")
        if p.dtype not in _DTYPES or not p.is_contiguous():
            raise TypeError("parameters must be contiguous float16 or float32")
    if group["copies"] is not None and len(group["copies"]) != len(group["params"]):
        raise ValueError("copies must hold a tensor or None for each parameter")
    if len({t.get_device() for t in (*group["params"], *(group["copies"] or ())) if t is not None}) > 1:
        raise ValueError("a group's parameters and copies must be on one GPU")
    _check_rates(group)


class _Plan:
    """A plan of the library with its workspace, and the tensors whose addresses it holds but the gradients: those are the
    program's to free when a step has been enqueued, and a plan is taken again only where they are at the same addresses."""

    def __init__(self, key, params, values, copies, states, device):
        self.key, self.held = key, (values, copies, states)
        # what a step writes and a program may have saved for a backward pass (inference tensors have no versions to count)
        self.written = [t for t in (*values, *copies) if t is not None and not t.is_inference()]
        self.workspace = torch.empty(fq.fq_adamw_workspace_bytes(params), dtype=torch.uint8, device=device)
        self.handle = fq.fq_adamw_create(params, self.workspace)
        weakref.finalize(self, fq.fq_adamw_destroy, self.handle)       # (at the latest while the library is still there)
        self.stream = torch.cuda.current_stream()

    def used_here(self, gradients):
        """What was allocated on another stream than the current one stays until that is done with it, too."""
        stream = torch.cuda.current_stream()
        if stream != self.stream:
            self.workspace.record_stream(stream)
        if stream != torch.cuda.default_stream():
            for g in gradients:                     # (nothing happens to one that is of this stream)
                g.record_stream(stream)


class AdamW(torch.optim.Optimizer):
    """Decoupled weight decay Adam over float16 and float32 parameters on one GPU.

    states: "float32" or "float8".  seed: of the stochastic rounding of float8 states.  A group may override lr, betas, eps,
    weight_decay and states, and may bring `copies`: one float16 tensor (or None) per float32 parameter, which receives
    its new values.  Gradients may be float16 or float32 (torch gives a float32 parameter a float16 gradient only where its
    grad_dtype says so).  Elements whose gradient is not finite are left as they are.  A group counts its steps; for a parameter whose
    first gradient comes later they count from that one on.  Steps in which it has none after that leave it as it is and do
    count.  A group in which no parameter has a gradient does not count the step, nor does any group count or make a step that is
    refused.
    """

    def __init__(self, params, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, states="float32", seed=0):
        self._plans = {}
        super().__init__(params, dict(lr=lr, betas=betas, eps=eps, weight_decay=weight_decay, states=states, seed=seed, step=0,
                                      copies=None))

    def add_param_group(self, group):
        super().add_param_group(group)
        group = self.param_groups[-1]
        try:
            _check_group(group)
            # (groups round differently: each has its own part of the seeds)
            group["seed"] = int(group["seed"]) + ((len(self.param_groups) - 1) << 32)
        except Exception:
            self.param_groups.pop()
            raise

    def _begin(self, p, group):
        """Makes the state of a parameter in front of its first step."""
        state = self.state[p]
        if group["step"]:
            state["late"] = group["step"]           # steps of the group before that
        if group["states"] == "float8":
            blocks = (p.numel() + 255) // 256
            for name in ("m", "v"):
                state[name] = torch.zeros(p.shape, dtype=torch.float8_e4m3fn, device=p.device)
                state[name + "_scale"] = torch.zeros(blocks, device=p.device)
        else:
            for name in ("m", "v"):
                state[name] = torch.zeros(p.shape, device=p.device)

    def _launches(self, index, group, grad_scale, made):
        """A launch for the parameters with a gradient, or, where some had their first one late, for those of each step number:
        [(plan, what fq_adamw_step takes, gradients)]."""
        params = group["params"]
        columns = [params, [p.grad for p in params], group["copies"] or [None] * len(params)]
        pick = lambda some: [[column[i] for i in some] for column in columns]      # noqa: E731
        if any(g is None for g in columns[1]):
            columns = pick([i for i, g in enumerate(columns[1]) if g is not None])
            if not columns[0]:
                return []
        states = [self.state[p] for p in columns[0]]
        if not all(states):
            for p, state in zip(columns[0], states):
                if not state:
                    made.append(p)
                    self._begin(p, group)
        columns.append(states)
        parts = {0: columns}
        if any("late" in state for state in states):
            places = {}
            for i, state in enumerate(states):
                places.setdefault(state.get("late", 0), []).append(i)
            parts = {late: pick(some) for late, some in places.items()}
        beta1, beta2 = group["betas"]
        return [(self._plan((index, late), group["weight_decay"], *part),
                 fq.FqAdamW(group["lr"], beta1, beta2, group["eps"], group["step"] + 1 - late, group["seed"], grad_scale), part[1])
                for late, part in parts.items()]

    def _plan(self, place, decay, params, grads, copies, states):
        tensors = [t for state in states for t in state.values()]
        if place[1]:
            tensors = [t for t in tensors if torch.is_tensor(t)]
        # All that the plan's table is made of.  Gradients are often at other addresses in every step: then it is made anew (88 tensors:
        # 400 to 670 us on the host; a plan that is taken again 73).
        try:
            if not all(map(torch.Tensor.is_contiguous, grads)):
                raise TypeError("gradients must be dense and contiguous")
            key = (decay, *(list(map(torch.Tensor.data_ptr, ts)) for ts in (params, grads, tensors)), list(map(torch.Tensor.numel, params)),
                   [p.dtype for p in params], [g.dtype for g in grads], [None if c is None else c.data_ptr() for c in copies])
        except RuntimeError:
            if all(g.layout is torch.strided for g in grads):
                raise
            raise TypeError("gradients must be dense and contiguous") from None
        plan = self._plans.get(place)
        if plan is None or plan.key != key:
            lists = [fq.FqParam.from_torch(p.detach(), g, s["m"], s["v"], s.get("m_scale"), s.get("v_scale"), p16=c, weight_decay=decay)
                     for p, g, c, s in zip(params, grads, copies, states)]
            plan = self._plans[place] = _Plan(key, lists, [p.detach() for p in params], copies, tensors, params[0].device)
        return plan

    @torch.no_grad()
    def step(self, closure=None, grad_scale=None):
        """grad_scale: one float32 on the GPU that all gradients are multiplied by, or None.  Not under graph capture."""
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        # Everything is looked at before anything is launched: a step that is refused moves no group, and does not count.
        launches, made = [], []
        try:
            for index, group in enumerate(self.param_groups):
                if group["params"]:
                    _check_rates(group)
                    if grad_scale is not None and grad_scale.get_device() != group["params"][0].get_device():
                        raise ValueError("grad_scale is not on the GPU of the group")
                    with torch.cuda.device(group["params"][0].device):
                        # (replays would repeat the step number and its random bits, and a table copied by a capture is read later)
                        if torch.cuda.is_current_stream_capturing():
                            raise RuntimeError("AdamW.step() cannot be captured into a graph; fq_adamw_step with a plan of its own can")
                        launches.append((group, self._launches(index, group, grad_scale, made)))
        except BaseException:
            for p in made:                          # (its first gradient is yet to come)
                del self.state[p]
            raise
        for group, parts in launches:
            with torch.cuda.device(group["params"][0].device):
                for plan, rates, gradients in parts:
                    plan.used_here(gradients)
                    fq.fq_adamw_step(plan.handle, rates)
                    torch.autograd.graph.increment_version(plan.written)
            if parts:
                group["step"] += 1
        return loss

    def __setstate__(self, state):
        super().__setstate__(state)
        self._plans = {}                            # (plans belong to the tensors of the optimizer that was copied or pickled)

    def state_dict(self):
        """Without the copies, which are the program's own and follow from the parameters."""
        packed = super().state_dict()
        for group in packed["param_groups"]:
            group["copies"] = None
        return packed

    def load_state_dict(self, state_dict):
        copies = [group["copies"] for group in self.param_groups]
        super().load_state_dict(state_dict)
        for group, own in zip(self.param_groups, copies):
            group["copies"] = own
        # The base class turns the states into the parameters' type.  They are codes, scales and floats: put back as saved.
        saved = [i for g in state_dict["param_groups"] for i in g["params"]]
        own = [p for g in self.param_groups for p in g["params"]]
        for i, p in zip(saved, own):
            if i in state_dict["state"]:
                self.state[p] = {k: v.to(p.device, copy=True) if torch.is_tensor(v) else v for k, v in state_dict["state"][i].items()}
        self._plans = {}
