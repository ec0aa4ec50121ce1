"""From a model's gradient tensors to the [K][d] rows of a step and back: the norm of many tensors, clipping by it,
packing (clipped on the way) and unpacking.  Methods mirror the `sae_grads_*` entry points of include/sae.h one to
one; argument checks and marshalling only, there is no CPU fallback.
"""
import ctypes as C
import math
from array import array

import numpy as np
import torch

from . import binding
from .binding import ABI_VERSION, NORM_MAX, NORM_NONE, NORM_ONE, NORM_TWO, OK, SaeError, SaeGradsConfig

TYPE_OF = {torch.float32: binding.TYPE_FLOAT, torch.bfloat16: binding.TYPE_BFLOAT, torch.float16: binding.TYPE_HALF}

_ptr, _numel, _dtype, _device, _dense = (torch.Tensor.data_ptr, torch.Tensor.numel, torch.Tensor.dtype.__get__,
                                         torch.Tensor.get_device, torch.Tensor.is_contiguous)


def _norm_kind(norm_type):
    kind = {2: NORM_TWO, 1: NORM_ONE, math.inf: NORM_MAX}.get(norm_type)
    if kind is None:
        raise ValueError("norm_type must be 1, 2 or inf")
    return kind


def _fills_its_span(t):
    """Whether t's elements lie without gaps or overlap, in whatever order."""
    want = 1
    for stride, size in sorted((st, n) for st, n in zip(t.stride(), t.shape) if n != 1):
        if stride != want:
            return False
        want *= size
    return True


class GradSet:
    """The plan of one parameter list: `num_rows` workers' gradients (or parameters) of T tensors each.

    tensor_sizes: elements of the T tensors; dtypes: one torch dtype for all or a list of T (float32, bfloat16,
    float16; default float32).  Tensors handed to a call are then contiguous.  `GradSet.like(tensors)` takes sizes,
    types and memory formats from a model's parameters instead: its tensors must have the strides of those (as
    autograd gives them: channels-last weights have channels-last gradients), and are packed in the order in which
    they lie in memory, the same for parameters and gradients.

    `tensors` of a call: T tensors (num_rows = 1) or num_rows lists of T; with T = 1 also one [num_rows, n] tensor.
    Work is enqueued on the stream the set was made on (or `stream`); a call made while another stream is current
    orders the two, so that tensors of the current stream can be handed over."""

    def __init__(self, num_rows, tensor_sizes, dtypes=None, device=None, stream=None, _strides=None):
        self.h = None
        sizes = np.ascontiguousarray(tensor_sizes, dtype=np.int64)
        self.K, self.T = int(num_rows), len(sizes)
        self.sizes = sizes.tolist()
        self.d = sum(self.sizes)
        if dtypes is None or isinstance(dtypes, torch.dtype):
            dtypes = [dtypes or torch.float32] * self.T
        self.dtypes = list(dtypes)
        if len(self.dtypes) != self.T or any(t not in TYPE_OF for t in self.dtypes):
            raise ValueError("dtypes: one of float32, bfloat16, float16 for every tensor")
        self.strides = _strides
        self.device = torch.device("cuda") if device is None else torch.device(device)
        if self.device.type != "cuda":
            raise ValueError("a gradient set lives on a CUDA device")
        index = torch.cuda.current_device() if self.device.index is None else self.device.index
        self.device = torch.device("cuda", index)
        self.devices = [index] * self.T
        self.stream = torch.cuda.current_stream(self.device).cuda_stream if stream is None else int(stream)
        types = np.array([TYPE_OF[t] for t in self.dtypes], dtype=np.int32)
        cfg = SaeGradsConfig(ABI_VERSION, self.K, self.T, sizes.ctypes.data_as(C.POINTER(C.c_int64)),
                             types.ctypes.data_as(C.POINTER(C.c_int32)), index, C.c_void_p(self.stream))
        h = C.c_void_p()
        self._check(binding.lib().sae_grads_init(C.byref(cfg), C.byref(h)), "sae_grads_init", None)
        self.h = h

    @classmethod
    def like(cls, tensors, num_rows=1, dtypes=None, stream=None):
        """The set of tensors shaped like `tensors` (a model's parameters); dtypes default to theirs."""
        tensors = list(tensors)
        if not tensors or not all(_fills_its_span(t) for t in tensors):
            raise ValueError("tensors must be dense: no gaps, no overlap")
        return cls(num_rows, [t.numel() for t in tensors], [t.dtype for t in tensors] if dtypes is None else dtypes,
                   tensors[0].device, stream, [(t.shape, t.stride()) for t in tensors])

    @staticmethod
    def _check(status, what, h):
        if status != OK:
            raise SaeError(status, what, binding.lib().sae_grads_last_cuda_error(h))

    def close(self):
        if self.h:
            binding.lib().sae_grads_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _row(self, row):
        if len(row) != self.T:
            raise ValueError(f"a row has {self.T} tensors, got {len(row)}")
        if list(map(_dtype, row)) != self.dtypes or list(map(_device, row)) != self.devices:
            raise ValueError("a tensor's dtype or device is not the set's")
        if self.strides is None:
            if list(map(_numel, row)) != self.sizes or not all(map(_dense, row)):
                raise ValueError("tensors must be contiguous and of the set's sizes")
        elif [(t.shape, t.stride()) for t in row] != self.strides:
            for t, (shape, stride) in zip(row, self.strides):      # strides of dimensions of one element are free
                if t.shape != shape or any(a != b for a, b, n in zip(t.stride(), stride, shape) if n != 1):
                    raise ValueError("tensors must have the shapes and strides that the set was made like")
        return map(_ptr, row)

    def _pointers(self, tensors):
        if isinstance(tensors, torch.Tensor):
            t = tensors
            if self.T != 1 or t.dim() != 2 or t.shape[0] != self.K or t.shape[1] != self.sizes[0] \
                    or (t.shape[1] > 1 and t.stride(1) != 1) or (self.K > 1 and t.stride(0) < t.shape[1]):
                raise ValueError("one tensor stands for [num_rows, n] of a set of one tensor, rows without gaps")
            if t.dtype != self.dtypes[0] or t.get_device() != self.devices[0]:
                raise ValueError("a tensor's dtype or device is not the set's")
            step = t.stride(0) * t.element_size()
            return array("Q", [t.data_ptr() + k * step for k in range(self.K)])
        if self.K == 1 and len(tensors) and isinstance(tensors[0], torch.Tensor):
            tensors = (tensors,)
        if len(tensors) != self.K:
            raise ValueError(f"tensors of {self.K} rows are wanted, got {len(tensors)}")
        out = array("Q")
        for row in tensors:
            out.extend(self._row(row))
        return out

    def _vector(self, v, what, same=False):
        """The row stride of a [d] (one row, or the same for all) or [num_rows, d] float32 tensor."""
        if not isinstance(v, torch.Tensor) or v.dtype != torch.float32 or v.get_device() != self.devices[0]:
            raise ValueError(f"{what} must be a float32 tensor on the set's device")
        if v.dim() == 1 and v.shape[0] == self.d and (self.K == 1 or same) and (self.d < 2 or v.stride(0) == 1):
            return 0
        if v.dim() == 2 and v.shape[0] == self.K and v.shape[1] == self.d and (self.d < 2 or v.stride(1) == 1) \
                and (self.K == 1 or v.stride(0) >= self.d):
            return v.stride(0) if self.K > 1 else 0
        raise ValueError(f"{what} must have {self.K} rows of {self.d} elements without gaps")

    def _call(self, name, *args):
        """One entry point, ordered after and before the current stream's work where that is another stream."""
        current = torch._C._cuda_getCurrentRawStream(self.devices[0])
        if current == self.stream:
            status = getattr(binding.lib(), name)(self.h, *args)
        else:
            mine, theirs = torch.cuda.ExternalStream(self.stream, self.device), torch.cuda.current_stream(self.device)
            mine.wait_stream(theirs)
            status = getattr(binding.lib(), name)(self.h, *args)
            theirs.wait_stream(mine)
        if status != OK:
            self._check(status, name, self.h)

    def _norms(self):
        return torch.empty(self.K, dtype=torch.float32, device=self.device)

    def norm(self, tensors, norm_type=2):
        """The norm of every row over all its tensors: float32 [num_rows], on the device."""
        kind, norms = _norm_kind(norm_type), self._norms()
        p = self._pointers(tensors)
        self._call("sae_grads_norm", p.buffer_info()[0], kind, norms.data_ptr())
        return norms

    def clip_(self, tensors, max_norm, norm_type=2):
        """Scales every row in place by min(1, max_norm / (norm + 1e-6)); returns the norms it had."""
        kind, norms = _norm_kind(norm_type), self._norms()
        p = self._pointers(tensors)
        self._call("sae_grads_clip", p.buffer_info()[0], kind, max_norm, norms.data_ptr())
        return norms

    def pack(self, tensors, out=None, max_norm=None, norm_type=2):
        """Concatenates every row's tensors into out ([num_rows, d] float32; [d] for one row), scaled by
        min(1, max_norm / (norm + 1e-6)) where max_norm is given.  Returns (out, norms or None)."""
        if out is None:
            out = torch.empty((self.K, self.d), dtype=torch.float32, device=self.device)
        stride = self._vector(out, "out")
        p = self._pointers(tensors)
        if max_norm is None:
            self._call("sae_grads_pack", p.buffer_info()[0], NORM_NONE, 0.0, out.data_ptr(), stride, None)
            return out, None
        kind, norms = _norm_kind(norm_type), self._norms()
        self._call("sae_grads_pack", p.buffer_info()[0], kind, max_norm, out.data_ptr(), stride, norms.data_ptr())
        return out, norms

    def unpack(self, vector, tensors):
        """Writes a [num_rows, d] vector's rows (or one [d] vector for every row) into the rows' tensors."""
        stride = self._vector(vector, "vector", same=True)
        p = self._pointers(tensors)
        self._call("sae_grads_unpack", vector.data_ptr(), stride, p.buffer_info()[0])
        return tensors
