"""Layers that stand between the aggregations of a model of node features: group norm with an activation, a gated
feed-forward block and the loss of a distillation from a teacher's best classes, each forward and backward in
hand-written kernels (include/da_layers.h).

float32 and bfloat16.  Each is one operation forward and one backward, in C++ (csrc/native_layers.cpp); this module
only checks and marshals arguments, and there is no fallback when the HIP library is missing (importing ``binding``
raises).  Work is enqueued on the current stream of the operands' device; the calls can be captured in a HIP graph.
Gradients cannot be differentiated again (asking for that raises).
"""
from __future__ import annotations

import torch

from . import _native
from . import binding as da

ACTIVATIONS = {None: da.DA_ACT_NONE, "relu": da.DA_ACT_RELU, "silu": da.DA_ACT_SILU, "gelu": da.DA_ACT_GELU,
               "sigmoid": da.DA_ACT_SIGMOID}


def _activation(name) -> int:
    try:
        return ACTIVATIONS[name]
    except (KeyError, TypeError):
        raise ValueError(f"activation must be one of {', '.join(map(repr, ACTIVATIONS))}, not {name!r}") from None


class _GroupNorm(torch.autograd.Function):
    """The operation where torch has more to do than backward differentiation: the Function supports or refuses it."""

    @staticmethod
    def forward(ctx, x, weight, bias, groups, eps, act, offsets):
        y, stats = _native.group_norm_forward(x, groups, weight, bias, eps, act, offsets)
        ctx.save_for_backward(x, weight, bias, offsets, stats)
        ctx.args = (groups, eps, act)
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        x, weight, bias, offsets, stats = ctx.saved_tensors
        groups, eps, act = ctx.args
        dx, dw, db = _native.group_norm_backward(dy, x, groups, weight, bias, eps, act, offsets, stats)
        return dx, dw, db, None, None, None, None


def group_norm(x: torch.Tensor, groups: int, weight: torch.Tensor | None = None, bias: torch.Tensor | None = None,
               eps: float = 1e-5, activation: str | None = None, offsets: torch.Tensor | None = None) -> torch.Tensor:
    """act(weight (x - mean) / sqrt(var + eps) + bias), channels last, mean and (biased) variance over the numbers that
    a sample has in a group of channels.

    x (..., L, C): every sample is L rows of C channels: (nodes, C) is one graph, (nodes, 1, C) normalises every node
    by itself.  With offsets, int32[samples + 1] on the device, x is (rows, C) and sample s is its rows offsets[s] up to
    offsets[s + 1]: a batch of graphs, empty ones allowed.  offsets are trusted to be well formed (from 0 to rows,
    non-decreasing), like the row pointers of a matrix, and left as they are until the backward pass.
    weight, bias: C numbers, float32 or bfloat16 whatever the type of x.  activation: None, "relu", "silu", "gelu", "sigmoid"."""
    act, eps, groups = _activation(activation), float(eps), int(groups)
    if _native.layers_take(x, weight, bias, offsets):
        return _native.group_norm(x, groups, weight, bias, eps, act, offsets)
    return _GroupNorm.apply(x, weight, bias, groups, eps, act, offsets)


class GroupNorm(torch.nn.Module):
    """group_norm with its parameters; forward takes the offsets of a batch of graphs."""

    def __init__(self, groups: int, channels: int, eps: float = 1e-5, activation: str | None = None, affine: bool = True):
        super().__init__()
        if groups < 1 or channels % groups:
            raise ValueError("channels must be a multiple of groups")
        _activation(activation)
        self.groups, self.eps, self.activation = groups, eps, activation
        self.weight = torch.nn.Parameter(torch.ones(channels)) if affine else None
        self.bias = torch.nn.Parameter(torch.zeros(channels)) if affine else None

    def forward(self, x: torch.Tensor, offsets: torch.Tensor | None = None) -> torch.Tensor:
        return group_norm(x, self.groups, self.weight, self.bias, self.eps, self.activation, offsets)


class _Gated(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w_gate, w_up, w_down, act):
        y, *kept = _native.gated_forward(x, w_gate, w_up, w_down, act)
        ctx.save_for_backward(x, w_gate, w_up, w_down, *kept)
        ctx.act = act
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        x, w_gate, w_up, w_down, *kept = ctx.saved_tensors
        return *_native.gated_backward(dy, x, w_gate, w_up, w_down, ctx.act, *kept), None


def gated_feed_forward(x: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor, w_down: torch.Tensor,
                       activation: str | None = "silu") -> torch.Tensor:
    """(act(x . w_gate) * (x . w_up)) . w_down for x (..., d), w_gate and w_up (d, h), w_down (h, d_out), all float32 or all
    bfloat16.  activation as for group_norm.  For the backward pass both projections are kept in float32 and their gated
    product in the type of x.  Weights whose rows are not dense (a transposed one, say) are copied at every call."""
    act = _activation(activation)
    if _native.layers_take(x, w_gate, w_up, w_down):
        return _native.gated(x, w_gate, w_up, w_down, act)
    return _Gated.apply(x, w_gate, w_up, w_down, act)


class GatedFeedForward(torch.nn.Module):
    """gated_feed_forward with its weights, (in, out) like those of GraphConv."""

    def __init__(self, features: int, hidden: int, out_features: int | None = None, activation: str | None = "silu"):
        super().__init__()
        _activation(activation)
        self.activation = activation
        self.w_gate = torch.nn.Parameter(torch.empty(features, hidden))
        self.w_up = torch.nn.Parameter(torch.empty(features, hidden))
        self.w_down = torch.nn.Parameter(torch.empty(hidden, features if out_features is None else out_features))
        for w in (self.w_gate, self.w_up, self.w_down):
            torch.nn.init.xavier_uniform_(w)

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        return gated_feed_forward(x, self.w_gate, self.w_up, self.w_down, self.activation)


class _Distill(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, top_index, top_logits, temperature):
        loss, stats = _native.distill_forward(logits, top_index, top_logits, temperature)
        ctx.save_for_backward(logits, top_index, top_logits, stats)
        ctx.temperature = temperature
        return loss

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dloss):
        logits, top_index, top_logits, stats = ctx.saved_tensors
        return _native.distill_backward(dloss, logits, stats, top_index, top_logits, ctx.temperature), None, None, None


def distill_loss(logits: torch.Tensor, top_index: torch.Tensor, top_logits: torch.Tensor, temperature: float = 1.0,
                 reduction: str = "mean") -> torch.Tensor:
    """temperature^2 KL(p || q), p the softmax of the teacher's best logits (over temperature), q the student's over all
    classes.

    logits (..., classes): the student's, differentiable.  top_index, top_logits (..., best): the teacher's best classes
    (int32 or int64; an entry outside 0 .. classes - 1, such as -1, is missing) and their logits (constants of the
    loss).  A row without entries has loss 0 and no gradient.  The loss is float32; reduction "none" gives one a row,
    "sum" their sum, "mean" that over the number of rows."""
    temperature = float(temperature)
    if not 0.0 < temperature < float("inf"):
        raise ValueError("temperature must be positive and finite")
    if reduction not in ("none", "sum", "mean"):
        raise ValueError(f"reduction must be 'none', 'sum' or 'mean', not {reduction!r}")
    if _native.layers_take(logits, top_index, top_logits):
        loss = _native.distill(logits, top_index, top_logits, temperature)
    else:
        loss = _Distill.apply(logits, top_index, top_logits, temperature)
    return loss if reduction == "none" else loss.sum() if reduction == "sum" else loss.mean()
