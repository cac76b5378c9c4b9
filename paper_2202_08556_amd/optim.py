"""Orthogonalised updates of weights: the momentum of a matrix's gradient, moved towards the nearest matrix with orthonormal
rows or columns, so that a step turns all directions of the weight alike (include/da_training.h; csrc/da_orthogonal.hip).

float32 and bfloat16 on the GPU, in hand-written kernels; there is no fallback when the HIP library is missing (importing
``binding`` raises).  Work is enqueued on the current stream of the operands' device; the calls can be captured in a HIP
graph.
"""
from __future__ import annotations

import torch

from . import _native
from . import binding as da  # noqa: F401  (loads the library)

# a, b, c of X <- a X + (b A + c A^2) X, A = X X^T: singular values between 0.01 and 1 come to 0.7 .. 1.2 in five steps
COEFFICIENTS = (3.4445, -4.775, 2.0315)
MATRICES = 65535                             # that a call takes


class _Orthogonalise(torch.autograd.Function):
    """The operation where torch has more to do than differentiate backwards: the Function supports or refuses it."""

    @staticmethod
    def forward(ctx, update, steps, coefficients, eps):
        return _native.orthogonalise(update, steps, coefficients, eps)

    @staticmethod
    def backward(ctx, dy):
        raise RuntimeError("orthogonalise has no gradient")


def orthogonalise(update: torch.Tensor, steps: int = 5, coefficients=COEFFICIENTS, eps: float = 1e-7) -> torch.Tensor:
    """Newton-Schulz steps X <- a X + (b A + c A^2) X, A = X X^T, from X = update / (|update| + eps) (Frobenius norm).

    update (..., rows, columns): each matrix by itself, the like weights of several layers at once; what is stacked costs less
    than one after the other.  coefficients: (a, b, c), or one such triple a step.  The products have 22 bits; a bfloat16
    result is rounded once, at the end.  Not differentiable: call it without gradients."""
    steps, eps = int(steps), float(eps)
    if steps < 0:
        raise ValueError("steps must not be negative")
    coefficients = list(coefficients)
    triples = coefficients if not coefficients or hasattr(coefficients[0], "__len__") else [coefficients] * steps
    if len(triples) != steps or any(len(t) != 3 for t in triples):
        raise ValueError("coefficients must be (a, b, c), or one such triple a step")
    if torch.is_grad_enabled() and update.requires_grad:
        raise ValueError("orthogonalise has no gradient: detach the update")
    flat = [float(v) for t in triples for v in t]
    if _native.layers_take(update):
        return _native.orthogonalise(update, steps, flat, eps)
    return _Orthogonalise.apply(update, steps, flat, eps)


class OrthogonalMomentum(torch.optim.Optimizer):
    """p <- (1 - lr weight_decay) p - lr max(1, outputs / inputs)^(1/2) orthogonalise(momentum of the gradient), for weights
    that are matrices (the last two axes); other parameters belong to another optimizer.  Weights of one shape and type are
    orthogonalised in one call, 65535 matrices at most.

    out_axis says which axis of a weight goes along its layer's outputs: -2, the rows, as in torch.nn.Linear, or -1 for weights
    (in, out) like those of GraphConv, GatedFeedForward and linear_cross_entropy.  It can differ by parameter group.

    The momentum is held in float32 whatever the weight's type, and rounded to that once for what is orthogonalised."""

    def __init__(self, params, lr: float = 0.02, momentum: float = 0.95, nesterov: bool = True, weight_decay: float = 0.0,
                 steps: int = 5, coefficients=COEFFICIENTS, eps: float = 1e-7, out_axis: int = -2):
        if lr < 0.0 or not 0.0 <= momentum < 1.0 or weight_decay < 0.0:
            raise ValueError("lr and weight_decay must not be negative, momentum in [0, 1)")
        super().__init__(params, dict(lr=lr, momentum=momentum, nesterov=nesterov, weight_decay=weight_decay, steps=steps,
                                      coefficients=coefficients, eps=eps, out_axis=out_axis))

    def __setstate__(self, state):
        super().__setstate__(state)
        for group in self.param_groups:                      # saved before there was a choice
            group.setdefault("out_axis", -2)

    def load_state_dict(self, state_dict):
        super().load_state_dict(state_dict)
        # torch rounds a state to the type of its parameter
        ids = [i for group in state_dict["param_groups"] for i in group["params"]]
        for i, p in zip(ids, [p for group in self.param_groups for p in group["params"]]):
            kept = state_dict["state"].get(i, {}).get("momentum")
            if kept is not None:
                self.state[p]["momentum"] = kept.detach().to(p.device, torch.float32, copy=True)

    def add_param_group(self, group):
        super().add_param_group(group)
        wrong = None
        if any(p.dim() < 2 for p in self.param_groups[-1]["params"]):
            wrong = "OrthogonalMomentum takes matrices; give vectors and numbers to another optimizer"
        elif self.param_groups[-1]["out_axis"] not in (-1, -2):
            wrong = "out_axis must be -2 (weights (out, in)) or -1 (weights (in, out))"
        if wrong:
            self.param_groups.pop()
            raise ValueError(wrong)

    @torch.no_grad()
    def step(self, closure=None):
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        for group in self.param_groups:
            alike: dict = {}
            for p in group["params"]:
                if p.grad is None:
                    continue
                state = self.state[p]
                if "momentum" not in state:
                    state["momentum"] = torch.zeros_like(p, dtype=torch.float32)
                m = state["momentum"].mul_(group["momentum"]).add_(p.grad)
                update = (p.grad.add(m, alpha=group["momentum"]) if group["nesterov"] else m).to(p.dtype)
                alike.setdefault((p.shape, p.dtype, p.device), []).append((p, update))
            for (shape, _, _), pairs in alike.items():
                most = max(1, MATRICES // max(1, shape[:-2].numel()))
                turned = []
                for k in range(0, len(pairs), most):
                    some = [u for _, u in pairs[k:k + most]]
                    many = torch.stack(some) if len(some) > 1 else some[0].unsqueeze(0)
                    turned += orthogonalise(many, group["steps"], group["coefficients"], group["eps"])
                outputs, inputs = shape[group["out_axis"]], shape[-3 - group["out_axis"]]
                size = group["lr"] * max(1.0, outputs / inputs) ** 0.5 if inputs else 0.0
                for (p, _), t in zip(pairs, turned):
                    if group["weight_decay"]:
                        p.mul_(1.0 - group["lr"] * group["weight_decay"])
                    p.add_(t, alpha=-size)
        return loss
