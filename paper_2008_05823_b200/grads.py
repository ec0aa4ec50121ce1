"""From a model's gradient tensors to the [K][d] rows of a step and back: the norm of many tensors, clipping by it,
packing (clipped on the way) and unpacking.  Methods mirror the `sae_grads_*` entry points of include/sae.h one to
one; what looks at the tensors is csrc/host_torch.cpp, and there is no CPU fallback.
"""
import ctypes as C
import math

import numpy as np
import torch

from . import binding
from .binding import ABI_VERSION, NORM_MAX, NORM_NONE, NORM_ONE, NORM_TWO, OK, SaeError, SaeGradsConfig

TYPE_OF = {torch.float32: binding.TYPE_FLOAT, torch.bfloat16: binding.TYPE_BFLOAT, torch.float16: binding.TYPE_HALF}


def _norm_kind(norm_type):
    kind = {2: NORM_TWO, 1: NORM_ONE, math.inf: NORM_MAX}.get(norm_type)
    if kind is None:
        raise ValueError("norm_type must be 1, 2 or inf")
    return kind


def _fills_its_span(t):
    """Whether t's elements lie without gaps or overlap, in whatever order."""
    if t.numel() == 0:
        return True
    want = 1
    for stride, size in sorted((st, n) for st, n in zip(t.stride(), t.shape) if n != 1):
        if stride != want:
            return False
        want *= size
    return True


class _Closed:
    """What a set has in place of its plan when it is closed: every call is refused."""

    def __getattr__(self, name):
        raise SaeError(binding.ERR_INVALID_ARG, f"{name} of a closed gradient set")


class GradSet:
    """The plan of one parameter list: `num_rows` workers' gradients (or parameters) of T tensors each.

    tensor_sizes: elements of the T tensors; dtypes: one torch dtype for all or a list of T (float32, bfloat16,
    float16; default float32).  Tensors handed to a call are then contiguous.  `GradSet.like(tensors)` takes sizes,
    types and memory formats from a model's parameters instead: its tensors must have the strides of those (as
    autograd gives them: channels-last weights have channels-last gradients), and are packed in the order in which
    they lie in memory, the same for parameters and gradients.

    `tensors` of a call: T tensors (num_rows = 1) or num_rows lists of T; with T = 1 also one [num_rows, n] tensor.
    What a call writes (clip_'s and unpack's tensors, pack's out) counts as changed in place: a backward pass that needs the
    old values raises.  Results take no part in autograd.
    Work is enqueued on the stream the set was made on (or `stream`); a call made while another stream is current
    orders the two, so that tensors of the current stream can be handed over."""

    def __init__(self, num_rows, tensor_sizes, dtypes=None, device=None, stream=None, _like=None):
        self.h, self._plan = None, _Closed()
        sizes = np.ascontiguousarray(tensor_sizes, dtype=np.int64)
        self.K, self.T = int(num_rows), len(sizes)
        self.sizes = sizes.tolist()
        self.d = sum(self.sizes)
        if dtypes is None or isinstance(dtypes, torch.dtype):
            dtypes = [dtypes or torch.float32] * self.T
        self.dtypes = list(dtypes)
        if len(self.dtypes) != self.T or any(t not in TYPE_OF for t in self.dtypes):
            raise ValueError("dtypes: one of float32, bfloat16, float16 for every tensor")
        self.device = torch.device("cuda") if device is None else torch.device(device)
        if self.device.type != "cuda":
            raise ValueError("a gradient set lives on a CUDA device")
        index = torch.cuda.current_device() if self.device.index is None else self.device.index
        self.device = torch.device("cuda", index)
        self.stream = torch.cuda.current_stream(self.device).cuda_stream if stream is None else int(stream)
        types = np.array([TYPE_OF[t] for t in self.dtypes], dtype=np.int32)
        cfg = SaeGradsConfig(ABI_VERSION, self.K, self.T, sizes.ctypes.data_as(C.POINTER(C.c_int64)),
                             types.ctypes.data_as(C.POINTER(C.c_int32)), index, C.c_void_p(self.stream))
        h = C.c_void_p()
        self._check(binding.lib().sae_grads_init(C.byref(cfg), C.byref(h)), "sae_grads_init", None)
        self.h = h
        self._plan = binding.host().GradPlan(h.value, self.K, self.sizes, types.tolist(), index, self.stream, _like or [])

    @classmethod
    def like(cls, tensors, num_rows=1, dtypes=None, stream=None):
        """The set of tensors shaped like `tensors` (a model's parameters); dtypes default to theirs."""
        tensors = list(tensors)
        if not tensors or not all(_fills_its_span(t) for t in tensors):
            raise ValueError("tensors must be dense: no gaps, no overlap")
        return cls(num_rows, [t.numel() for t in tensors], [t.dtype for t in tensors] if dtypes is None else dtypes,
                   tensors[0].device, stream, [(list(t.shape), list(t.stride())) for t in tensors])

    @staticmethod
    def _check(status, what, h):
        if status != OK:
            raise SaeError(status, what, binding.lib().sae_grads_last_cuda_error(h))

    def close(self):
        if self.h:
            self._plan = _Closed()
            binding.lib().sae_grads_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def norm(self, tensors, norm_type=2):
        """The norm of every row over all its tensors: float32 [num_rows], on the device."""
        status, norms = self._plan.norm(tensors, _norm_kind(norm_type))
        if status:
            self._check(status, "sae_grads_norm", self.h)
        return norms

    def clip_(self, tensors, max_norm, norm_type=2):
        """Scales every row in place by min(1, max_norm / (norm + 1e-6)), rounded to each tensor's type as torch's own
        in-place product does; returns the norms it had."""
        status, norms = self._plan.clip(tensors, _norm_kind(norm_type), max_norm)
        if status:
            self._check(status, "sae_grads_clip", self.h)
        return norms

    def pack(self, tensors, out=None, max_norm=None, norm_type=2):
        """Concatenates every row's tensors into out ([num_rows, d] float32; [d] for one row), scaled by
        min(1, max_norm / (norm + 1e-6)) where max_norm is given.  Returns (out, norms or None)."""
        kind = NORM_NONE if max_norm is None else _norm_kind(norm_type)
        status, out, norms = self._plan.pack(tensors, out, kind, 0.0 if max_norm is None else max_norm)
        if status:
            self._check(status, "sae_grads_pack", self.h)
        return out, norms

    def unpack(self, vector, tensors):
        """Writes a [num_rows, d] vector's rows (or one [d] vector for every row) into the rows' tensors."""
        status = self._plan.unpack(vector, tensors)
        if status:
            self._check(status, "sae_grads_unpack", self.h)
        return tensors
