"""Linear cross entropy: the loss of a linear output layer over its classes, and its gradients, with no logits kept.
`linear_cross_entropy` (differentiable), the `LinearCrossEntropy` module, and the two calls under them,
`linear_cross_entropy_forward` and `linear_cross_entropy_backward`, which mirror the entry points of include/sae.h.  What looks
at the tensors is csrc/host_torch.cpp; there is no CPU fallback.
"""
import math

import torch

from . import binding
from .binding import SaeError

REDUCTION_OF = {"none": binding.REDUCE_NONE, "sum": binding.REDUCE_SUM, "mean": binding.REDUCE_MEAN}


def _reduction(name):
    if name not in REDUCTION_OF:
        raise ValueError(f"reduction must be one of {', '.join(REDUCTION_OF)}")
    return REDUCTION_OF[name]


def linear_cross_entropy_forward(x, weight, target, bias=None, ignore_index=-100, reduction="mean"):
    """The cross entropy of x @ weight.T + bias ([..., classes], not kept) against target [...].
    Returns (loss, lse, count): the loss in float32, of target's shape for "none"; the logarithm of every row's sum of
    exponentials, 0 for a row whose target is ignore_index; the number of the other rows, int64.
    lse.rest is what rounding to float32 left out of lse: the backward call reads it.  A copy of lse does not have it."""
    loss, lse, rest, count = _forward(x, weight, target, bias, ignore_index, reduction)
    lse.rest = rest
    return loss, lse, count


def _forward(x, weight, target, bias, ignore_index, reduction):
    status, *out = binding.host().linear_ce_forward(x, weight, target, bias, ignore_index, _reduction(reduction))
    if status:
        raise SaeError(status, "sae_linear_ce_forward")
    return out


def linear_cross_entropy_backward(dloss, x, weight, target, lse, count, bias=None, ignore_index=-100, reduction="mean",
                                  need_x=True, need_weight=True, need_bias=True):
    """The gradients of linear_cross_entropy_forward's loss: (dx, dweight, dbias), None where there is no such input or it is not
    wanted.  lse and count are what the forward call returned; with a copy of lse the rows' sums are made again, for a fourth more work.
    dloss is float32, of the loss's shape."""
    return _backward(dloss, x, weight, target, lse, getattr(lse, "rest", None), count, bias, ignore_index, reduction, need_x, need_weight, need_bias)


def _backward(dloss, x, weight, target, lse, rest, count, bias, ignore_index, reduction, need_x, need_weight, need_bias):
    status, *out = binding.host().linear_ce_backward(dloss, x, weight, target, lse, rest, count, bias, ignore_index, _reduction(reduction),
                                                     need_x, need_weight, need_bias)
    if status:
        raise SaeError(status, "sae_linear_ce_backward")
    return tuple(out)


class _LinearCrossEntropy(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, target, ignore_index, reduction):
        loss, lse, rest, count = _forward(x, weight, target, bias, ignore_index, reduction)
        ctx.save_for_backward(x, weight, bias, target, lse, rest, count)
        ctx.ignore_index, ctx.reduction = ignore_index, reduction
        return loss

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dloss):
        x, weight, bias, target, lse, rest, count = ctx.saved_tensors
        need = ctx.needs_input_grad
        return _backward(dloss, x, weight, target, lse, rest, count, bias, ctx.ignore_index, ctx.reduction,
                         need[0], need[1], need[2]) + (None, None, None)


def linear_cross_entropy(x, weight, target, bias=None, ignore_index=-100, reduction="mean"):
    """Differentiable cross entropy of x @ weight.T + bias against target; gradients of x, weight and bias.  Under autocast
    x and weight are taken in its type, as a linear layer takes them."""
    if torch.is_autocast_enabled("cuda"):
        kind = torch.get_autocast_dtype("cuda")
        x, weight = x.to(kind), weight.to(kind)
    return _LinearCrossEntropy.apply(x, weight, bias, target, ignore_index, reduction)


class LinearCrossEntropy(torch.nn.Module):
    """A linear output layer together with its cross entropy: the parameters of torch.nn.Linear(in_features, num_classes, bias),
    forward(x, target) gives the loss.  `logits(x)` is the layer alone, for predictions."""

    def __init__(self, in_features, num_classes, bias=True, ignore_index=-100, reduction="mean", device=None, dtype=None):
        super().__init__()
        if in_features < 1 or num_classes < 1:
            raise ValueError("in_features and num_classes must be at least 1")
        _reduction(reduction)
        self.in_features, self.num_classes, self.ignore_index, self.reduction = in_features, num_classes, ignore_index, reduction
        self.weight = torch.nn.Parameter(torch.empty(num_classes, in_features, device=device, dtype=dtype))
        self.bias = torch.nn.Parameter(torch.empty(num_classes, device=device, dtype=dtype)) if bias else None
        self.reset_parameters()

    def reset_parameters(self):
        bound = 1 / math.sqrt(self.in_features)
        torch.nn.init.uniform_(self.weight, -bound, bound)
        if self.bias is not None:
            torch.nn.init.uniform_(self.bias, -bound, bound)

    def forward(self, x, target):
        return linear_cross_entropy(x, self.weight, target, self.bias, self.ignore_index, self.reduction)

    def logits(self, x):
        return torch.nn.functional.linear(x, self.weight, self.bias)

    def extra_repr(self):
        return f"{self.in_features}, {self.num_classes}, bias={self.bias is not None}, reduction={self.reduction}"
