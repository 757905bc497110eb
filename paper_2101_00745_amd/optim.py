"""Optimisers: momentum whose update is orthogonalised, for the weight matrices of SCC layers (over scc_orthogonal_step), and AdamW for all other
weights (over scc_adamw_step)."""
import torch

from . import scc as _scc


class OrthogonalMomentum(torch.optim.Optimizer):
    """m <- momentum m + g; w <- (1 - lr weight_decay) w - lr sqrt(max(1, rows/cols)) O(g + momentum m), O five Newton-Schulz steps, which bring
    the singular values near 1 (``scc_orthogonal_step``).  Takes weights of two dimensions, or of three as a stack of matrices (the
    gate's and the other's of a ``GatedSCC``); everything else (biases, depthwise filters) is refused and belongs to another optimiser.  All matrices
    of a group and dtype are updated by one call; the momenta are float32."""

    def __init__(self, params, lr=0.02, momentum=0.95, weight_decay=0.0, nesterov=True, steps=5):
        if lr < 0.0 or not 0.0 <= momentum < 1.0 or weight_decay < 0.0 or steps < 1:
            raise ValueError("lr and weight_decay must not be negative, momentum must lie in [0, 1), steps must be at least 1")
        super().__init__(params, dict(lr=lr, momentum=momentum, weight_decay=weight_decay, nesterov=nesterov, steps=steps))

    def add_param_group(self, param_group):
        """Groups of the constructor come through here as well.  A stack of 3 x 3 matrices has the shape of depthwise filters, [C, 3, 3], and is
        taken for those."""
        super().add_param_group(param_group)
        for p in self.param_groups[-1]["params"]:
            if p.dim() not in (2, 3) or (p.dim() == 3 and tuple(p.shape[1:]) == (3, 3)):
                self.param_groups.pop()
                raise ValueError("weights must be matrices or stacks of matrices, and no depthwise filters [C, 3, 3]; got %s" % (tuple(p.shape),))

    def load_state_dict(self, state_dict):
        super().load_state_dict(state_dict)
        # torch brings a state to its parameter's type; the momenta of bfloat16 weights stay what they were
        saved = {i: s["momentum"] for i, s in state_dict["state"].items() if "momentum" in s}
        indices = [i for group in state_dict["param_groups"] for i in group["params"]]
        params = [p for group in self.param_groups for p in group["params"]]
        for i, p in zip(indices, params):
            if i in saved:
                self.state[p]["momentum"] = saved[i].to(device=p.device, dtype=torch.float32, copy=True)

    @torch.no_grad()
    def step(self, closure=None):
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        for group in self.param_groups:
            lists = {}
            for p in group["params"]:
                if p.grad is None:
                    continue
                state = self.state[p]
                if "momentum" not in state:
                    state["momentum"] = torch.zeros_like(p, dtype=torch.float32, memory_format=torch.contiguous_format)
                ws, gs, ms = lists.setdefault((p.device, p.dtype), ([], [], []))
                for to, t in ((ws, p), (gs, p.grad.contiguous()), (ms, state["momentum"])):
                    to.extend([t] if t.dim() == 2 else t.unbind(0))
            for ws, gs, ms in lists.values():
                _scc.scc_orthogonal_step(ws, gs, ms, group["lr"], momentum=group["momentum"], weight_decay=group["weight_decay"],
                                         nesterov=group["nesterov"], steps=group["steps"])
        return loss


class AdamW(torch.optim.Optimizer):
    """AdamW for the weights that ``OrthogonalMomentum`` does not take, or for all (``scc_adamw_step``): one call, in launches of 60 weights, for all weights of
    a group, dtype and age.  state_bits: 32, or 8 for states of e4m3 with a scale for each 256 elements, rounded at random (a hash of ``seed``, the
    step and the place, so that a run repeats; lists of one step round by the same numbers).  capturable: the step's number is kept on the GPU, so that a captured
    step can be replayed; make one step before the capture, which allocates the states.  A replay has the lr, betas, eps and weight_decay of the capture: where a
    schedule moves them, capture again.  bfloat16 weights are rounded to nearest: a step of less than half of theirs (2^-9 to 2^-8 of a weight; around
    1 that is two to four of the default lr) leaves them where they are."""

    def __init__(self, params, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, state_bits=32, seed=0, capturable=False):
        if lr < 0.0 or not all(0.0 <= b < 1.0 for b in betas) or eps < 0.0 or weight_decay < 0.0:
            raise ValueError("lr, eps and weight_decay must not be negative, betas must lie in [0, 1)")
        if state_bits not in (8, 32):
            raise ValueError("state_bits must be 8 or 32, got %r" % (state_bits,))
        super().__init__(params, dict(lr=lr, betas=tuple(betas), eps=eps, weight_decay=weight_decay, state_bits=state_bits, seed=int(seed),
                                      capturable=bool(capturable)))

    def load_state_dict(self, state_dict):
        super().load_state_dict(state_dict)
        # torch brings a state to its parameter's type; these stay what they were
        indices = [i for group in state_dict["param_groups"] for i in group["params"]]
        params = [p for group in self.param_groups for p in group["params"]]
        for i, p in zip(indices, params):
            for name, value in state_dict["state"].get(i, {}).items():
                if isinstance(value, torch.Tensor):
                    self.state[p][name] = value.to(device=p.device, copy=True)
        for group in self.param_groups:
            for p in group["params"]:
                step = self.state[p].get("step") if p in self.state else None
                if isinstance(step, torch.Tensor):
                    self.state[p]["step"] = self._shared_step(group, p.device, int(step), step)

    def _shared_step(self, group, device, age, step):
        """The weights of a group that are equally old share their step's number, where it is on the GPU: one call takes them all."""
        for p in group["params"]:
            other = self.state[p].get("step") if p in self.state else None
            if isinstance(other, torch.Tensor) and other is not step and other.device == device and int(other) == age:
                return other
        return step

    def _begin(self, p, group, begun, fresh):
        """The weight's state; begun: the numbers on the GPU of the weights that begin in this step; fresh: gets the weights whose states are made here."""
        state = self.state[p]
        if not state:
            fresh.append(p)
            if group["capturable"]:
                if p.device not in begun:
                    begun[p.device] = torch.zeros((), dtype=torch.int64, device=p.device)
                state["step"] = begun[p.device]
            else:
                state["step"] = 0
            if group["state_bits"] == 8:
                blocks = -(-p.numel() // _scc.STATE_BLOCK)
                for name in ("first", "second"):
                    state[name] = torch.zeros(p.shape, dtype=torch.uint8, device=p.device).view(torch.float8_e4m3fn)
                    state[name + "_scales"] = torch.ones(blocks, dtype=torch.float32, device=p.device)
            else:
                for name in ("first", "second"):
                    state[name] = torch.zeros(p.shape, dtype=torch.float32, device=p.device)
        return state

    def _gather(self, group, moving, fresh):
        """The lists of the group's calls, each of one device, type, width of states and age: [weights, gradients, states and their scales]."""
        lists, begun = {}, {}
        for p in moving:
            state = self._begin(p, group, begun, fresh)
            step, scales = state["step"], [state.get("first_scales"), state.get("second_scales")]
            key = (p.device, p.dtype, scales[0] is None, id(step) if isinstance(step, torch.Tensor) else step)
            own = lists.setdefault(key, ([], [], [], [], *([None] * 2 if scales[0] is None else ([], []))))
            for to, t in zip(own, (p, p.grad.contiguous(), state["first"], state["second"], *scales)):
                if to is not None:
                    to.append(t)
        return list(lists.values())

    def _age(self, moving, by):
        seen = set()
        for p in moving:
            state = self.state[p]
            step = state["step"]
            if not isinstance(step, torch.Tensor):
                state["step"] = step + by
            elif id(step) not in seen:
                seen.add(id(step))
                step.add_(by)

    def _resting(self, group):
        """The numbers on the GPU of the weights that have no gradient in this step."""
        steps = (self.state[p].get("step") for p in group["params"] if p.grad is None and p in self.state)
        return {id(step) for step in steps if isinstance(step, torch.Tensor)}

    def _part(self, group, moving):
        """Weights that have aged together and of which some rest now: the others go on with a number of their own."""
        resting, fresh = self._resting(group), {}
        for p in moving if resting else ():
            step = self.state[p].get("step")
            if id(step) in resting:
                if id(step) not in fresh:
                    fresh[id(step)] = step.clone()
                self.state[p]["step"] = fresh[id(step)]

    def _check_capture(self, group, moving):
        """A replay repeats what the captured call did: it neither counts on the host nor makes states."""
        if not group["capturable"] or any(not isinstance(self.state.get(p, {}).get("step"), torch.Tensor) for p in moving):
            raise RuntimeError("a captured step wants capturable=True, and a step of the same weights before the capture")
        resting = self._resting(group)
        if any(id(self.state[p]["step"]) in resting for p in moving):
            raise RuntimeError("make a step with gradients for the same weights before the capture")

    @torch.no_grad()
    def step(self, closure=None):
        """Every call is looked at before one is made (the first one by itself: it is refused before it moves anything), so that a step that is refused leaves
        ages, weights and states as they were."""
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        groups = [(group, [p for p in group["params"] if p.grad is not None and p.numel()]) for group in self.param_groups]
        if any(p.is_cuda for _, moving in groups for p in moving) and torch.cuda.is_current_stream_capturing():
            for group, moving in groups:
                if moving:
                    self._check_capture(group, moving)
        fresh, raised = [], False
        try:
            calls = [(group, lists) for group, moving in groups for lists in self._gather(group, moving, fresh)]
            for group, lists in calls[1:]:
                _scc._refuse_adamw(*lists, group["lr"], self.state[lists[0][0]]["step"], group["betas"], group["eps"], group["weight_decay"])
            for group, moving in groups:
                self._part(group, moving)
                self._age(moving, 1)
            raised = True
            for i, (group, (ws, gs, ms, vs, mss, vss)) in enumerate(calls):
                _scc.scc_adamw_step(ws, gs, ms, vs, group["lr"], self.state[ws[0]]["step"], betas=group["betas"], eps=group["eps"],
                                    weight_decay=group["weight_decay"], first_scales=mss, second_scales=vss, seed=group["seed"])
        except Exception as e:
            if not raised or (i == 0 and getattr(e, "status", None) != _scc.SCC_ERR_LAUNCH):
                for _, moving in groups if raised else ():
                    self._age(moving, -1)
                for p in fresh:
                    del self.state[p]
            raise
        return loss
