"""Group norm with an activation, channels last: `group_norm` (differentiable), the `GroupNorm` module, and the two calls
under them, `group_norm_forward` and `group_norm_backward`, which mirror the entry points of include/sae.h.  Argument
checks and marshalling only; there is no CPU fallback.
"""
import ctypes as C

import torch

from . import binding
from .binding import OK, SaeError, SaeGroupNormDesc
from .grads import TYPE_OF

ACT_OF = {"none": binding.ACT_NONE, "relu": binding.ACT_RELU, "silu": binding.ACT_SILU, "gelu": binding.ACT_GELU}


def _strides(t, what):
    """(sample, pixel) strides of an [n, c, *space] tensor whose channels are neighbours in memory and whose pixels
    follow one another at one stride."""
    shape, st = t.shape, t.stride()
    if shape[1] > 1 and st[1] != 1:
        raise ValueError(f"{what} must be channels last: neighbouring channels next to each other in memory")
    pixel, run = 0, 1
    for size, stride in zip(reversed(shape[2:]), reversed(st[2:])):
        if size == 1:
            continue
        if run == 1:
            pixel = stride
        elif stride != run * pixel:
            raise ValueError(f"{what}: the pixels of a sample must follow one another at one stride")
        run *= size
    return (st[0] if shape[0] > 1 else 0), pixel


def _input(t, like, what):
    if not isinstance(t, torch.Tensor) or t.shape != like.shape or t.dtype != like.dtype or t.device != like.device:
        raise ValueError(f"{what} must have the shape, dtype and device of x")
    return _strides(t, what) if t.numel() else (0, 0)


def _describe(x, groups, weight, bias, eps, activation, residual, dy=None):
    if not isinstance(x, torch.Tensor) or not x.is_cuda or x.dtype not in TYPE_OF or x.dim() < 2:
        raise ValueError("x must be a float32, bfloat16 or float16 CUDA tensor [n, c, *space]")
    n, c = x.shape[0], x.shape[1]
    if groups < 1 or c < 1 or c % groups:
        raise ValueError("the number of groups must divide the number of channels")
    if activation not in ACT_OF:
        raise ValueError(f"activation must be one of {', '.join(ACT_OF)}")
    param = torch.float32
    for t, what in ((weight, "weight"), (bias, "bias")):
        if t is not None:
            if t.shape != (c,) or t.dtype not in TYPE_OF or t.device != x.device or not t.is_contiguous():
                raise ValueError(f"{what} must be a contiguous [c] tensor on x's device")
            param = t.dtype
    if weight is not None and bias is not None and weight.dtype != bias.dtype:
        raise ValueError("weight and bias must have the same dtype")
    xs = _input(x, x, "x")
    rs = _input(residual, x, "residual") if residual is not None else (0, 0)
    ds = _input(dy, x, "dy") if dy is not None else (0, 0)
    pixels = 1
    for s in x.shape[2:]:
        pixels *= s
    return SaeGroupNormDesc(TYPE_OF[x.dtype], TYPE_OF[param], ACT_OF[activation], groups, n, pixels, c, *xs, *rs, *ds, eps)


def _dense(x):
    """A new tensor of x's shape, channels last without gaps."""
    n, c, *space = x.shape
    return torch.empty((n, *space, c), dtype=x.dtype, device=x.device).movedim(-1, 1)


def _workspace(desc, x):
    size = binding.lib().sae_group_norm_workspace(C.byref(desc))
    if size < 0:
        raise SaeError(binding.ERR_INVALID_ARG, "sae_group_norm_workspace")
    return torch.empty(size, dtype=torch.uint8, device=x.device), size


def _ptr(t):
    return None if t is None else t.data_ptr()


def group_norm_forward(x, num_groups, weight=None, bias=None, eps=1e-5, activation="none", residual=None):
    """act(group_norm(x) * weight + bias (+ residual)) of x [n, c, *space], channels last in memory.
    Returns (y, mean, rstd); the statistics are float32 [n, groups]."""
    desc = _describe(x, num_groups, weight, bias, eps, activation, residual)
    with torch.cuda.device(x.device):
        y = _dense(x)
        mean = torch.empty((x.shape[0], num_groups), dtype=torch.float32, device=x.device)
        rstd = torch.empty_like(mean)
        ws, size = _workspace(desc, x)
        rc = binding.lib().sae_group_norm_forward(C.byref(desc), x.data_ptr(), _ptr(residual), _ptr(weight), _ptr(bias), y.data_ptr(),
                                                  mean.data_ptr(), rstd.data_ptr(), ws.data_ptr(), size,
                                                  torch._C._cuda_getCurrentRawStream(x.device.index))
    if rc != OK:
        raise SaeError(rc, "sae_group_norm_forward")
    return y, mean, rstd


def group_norm_backward(dy, x, mean, rstd, num_groups, weight=None, bias=None, activation="none", residual=None,
                        need_residual=True, need_params=True):
    """The gradients of group_norm_forward's y: (dx, dresidual, dweight, dbias), None where there is no such input or it
    is not wanted.  mean and rstd are what the forward call returned."""
    desc = _describe(x, num_groups, weight, bias, 0.0, activation, residual, dy)
    for t, what in ((mean, "mean"), (rstd, "rstd")):
        if t.shape != (x.shape[0], num_groups) or t.dtype != torch.float32 or t.device != x.device or not t.is_contiguous():
            raise ValueError(f"{what} must be the float32 [n, groups] tensor of the forward call")
    with torch.cuda.device(x.device):
        dx = _dense(x)
        dres = _dense(x) if residual is not None and need_residual else None
        dweight = torch.empty_like(weight) if weight is not None and need_params else None
        dbias = torch.empty_like(bias) if bias is not None and need_params else None
        ws, size = _workspace(desc, x)
        rc = binding.lib().sae_group_norm_backward(C.byref(desc), dy.data_ptr(), x.data_ptr(), _ptr(residual), mean.data_ptr(), rstd.data_ptr(),
                                                   _ptr(weight), _ptr(bias), dx.data_ptr(), _ptr(dres), _ptr(dweight), _ptr(dbias),
                                                   ws.data_ptr(), size, torch._C._cuda_getCurrentRawStream(x.device.index))
    if rc != OK:
        raise SaeError(rc, "sae_group_norm_backward")
    return dx, dres, dweight, dbias


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
        try:
            _strides(dy, "dy")
        except ValueError:                       # a gradient in another order: laid out like x
            dy = _dense(x).copy_(dy)
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
