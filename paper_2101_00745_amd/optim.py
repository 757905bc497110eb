"""Optimiser over scc_orthogonal_step: momentum whose update is orthogonalised, for the weight matrices of SCC layers."""
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
