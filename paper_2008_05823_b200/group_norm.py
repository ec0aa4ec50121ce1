"""Group norm with an activation, channels last: `group_norm` (differentiable), the `GroupNorm` module, and the two calls
under them, `group_norm_forward` and `group_norm_backward`, which mirror the entry points of include/sae.h.  What looks at
the tensors is csrc/host_torch.cpp; there is no CPU fallback.
"""
import torch

from . import binding
from .binding import SaeError

ACT_OF = {"none": binding.ACT_NONE, "relu": binding.ACT_RELU, "silu": binding.ACT_SILU, "gelu": binding.ACT_GELU}


def _act(name):
    if name not in ACT_OF:
        raise ValueError(f"activation must be one of {', '.join(ACT_OF)}")
    return ACT_OF[name]


def group_norm_forward(x, num_groups, weight=None, bias=None, eps=1e-5, activation="none", residual=None):
    """act(group_norm(x) * weight + bias (+ residual)) of x [n, c, *space], channels last in memory.
    Returns (y, mean, rstd); the statistics are float32 [n, groups]."""
    status, y, mean, rstd = binding.host().group_norm_forward(x, num_groups, weight, bias, eps, _act(activation), residual)
    if status:
        raise SaeError(status, "sae_group_norm_forward")
    return y, mean, rstd


def group_norm_backward(dy, x, mean, rstd, num_groups, weight=None, bias=None, activation="none", residual=None,
                        need_residual=True, need_params=True):
    """The gradients of group_norm_forward's y: (dx, dresidual, dweight, dbias), None where there is no such input or it
    is not wanted.  mean and rstd are what the forward call returned."""
    status, dx, dres, dweight, dbias = binding.host().group_norm_backward(dy, x, mean, rstd, num_groups, weight, bias, _act(activation),
                                                                          residual, need_residual, need_params)
    if status:
        raise SaeError(status, "sae_group_norm_backward")
    return dx, dres, dweight, dbias


def _channels_last(t):
    """Whether t has the layout that the calls take for granted, without gaps; other accepted ones are copied needlessly."""
    return t.movedim(1, -1).is_contiguous()


class _GroupNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, residual, num_groups, eps, activation):
        y, mean, rstd = group_norm_forward(x, num_groups, weight, bias, eps, activation, residual)
        ctx.save_for_backward(x, weight, bias, residual if activation != "none" else None, mean, rstd)
        ctx.num_groups, ctx.activation, ctx.has_residual = num_groups, activation, residual is not None
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        x, weight, bias, residual, mean, rstd = ctx.saved_tensors
        need = ctx.needs_input_grad
        if not _channels_last(dy):                          # a gradient in another order: laid out like x
            dy = dy.movedim(1, -1).contiguous().movedim(-1, 1)
        dx, dres, dweight, dbias = group_norm_backward(dy, x, mean, rstd, ctx.num_groups, weight, bias, ctx.activation, residual,
                                                       need[3], need[1] or need[2])
        if ctx.has_residual and ctx.activation == "none":
            dres = dy                            # z is y
        return dx if need[0] else None, dweight if need[1] else None, dbias if need[2] else None, dres if need[3] else None, None, None, None


def group_norm(x, num_groups, weight=None, bias=None, eps=1e-5, activation="none", residual=None):
    """Differentiable act(group_norm(x) * weight + bias (+ residual)), channels last; gradients of x, weight, bias, residual."""
    return _GroupNorm.apply(x, weight, bias, residual, num_groups, eps, activation)


class GroupNorm(torch.nn.Module):
    """Group norm with an activation over [n, c, *space] tensors that lie channels last; two parameter vectors, as a batch
    norm of the same layer has.  forward(x, residual=None) adds the residual before the activation."""

    def __init__(self, num_groups, num_channels, eps=1e-5, activation="none", device=None, dtype=None):
        super().__init__()
        if num_groups < 1 or num_channels % num_groups:
            raise ValueError("the number of groups must divide the number of channels")
        if activation not in ACT_OF:
            raise ValueError(f"activation must be one of {', '.join(ACT_OF)}")
        self.num_groups, self.num_channels, self.eps, self.activation = num_groups, num_channels, eps, activation
        self.weight = torch.nn.Parameter(torch.ones(num_channels, device=device, dtype=dtype))
        self.bias = torch.nn.Parameter(torch.zeros(num_channels, device=device, dtype=dtype))

    def forward(self, x, residual=None):
        return group_norm(x, self.num_groups, self.weight, self.bias, self.eps, self.activation, residual)

    def extra_repr(self):
        return f"{self.num_groups}, {self.num_channels}, eps={self.eps}, activation={self.activation}"
