"""Orthogonalisation of a model's matrices by Newton-Schulz products, all of them in one call: what a worker may do to its
gradients or its model difference before they are packed.  (The momentum of Sae.step lies behind that.  A momentum that is to be made orthogonal is kept
outside, and the step is made with momentum 0.)  `Orthogonalizer` mirrors the `sae_ortho_*` entry points of
include/sae.h; what looks at the tensors is csrc/host_torch.cpp, and there is no CPU fallback.
"""
import ctypes as C
import math

import numpy as np
import torch

from . import binding
from .binding import ABI_VERSION, ERR_INVALID_ARG, OK, SaeError, SaeOrthoConfig
from .grads import TYPE_OF

# Five steps of these bring every singular value above about 0.01 of the norm to within 0.7 .. 1.2 (a published choice: K. Jordan et al., "Muon: an optimizer
# for hidden layers in neural networks", 2024).
COEFFICIENTS = (3.4445, -4.7750, 2.0315)


class _Closed:
    def run(self, *_):
        raise SaeError(ERR_INVALID_ARG, "a call of a closed orthogonaliser")


def _per_matrix(value, count, what):
    kinds = [value] * count if isinstance(value, torch.dtype) else list(value)
    if len(kinds) != count or any(k not in TYPE_OF for k in kinds):
        raise ValueError(f"{what}: one of float32, bfloat16, float16 for every matrix")
    return kinds


class Orthogonalizer:
    """The plan of one list of matrices: `num_rows` workers' lists of T tensors each.

    x = g / (|g| + eps), then `steps` times x <- a x + b (x x') x + c (x x')^2 x: the same singular vectors, singular
    values driven towards 1.  A tensor of more than two dimensions is the matrix [first, all others] (a convolution's weight),
    whatever the order in which the others lie in memory; the result lies in the same order.

    shapes: of the T tensors; dtypes: one torch dtype or a list of T (float32, bfloat16, float16); result_dtypes: likewise, default
    dtypes.  coefficients: (a, b, c), or one such triple for every step.  `Orthogonalizer.like(tensors)` takes shapes and types
    from a model's parameters.

    plan(tensors, results=None): T tensors (num_rows = 1) or num_rows lists of T; returns results, new tensors where none are
    given.  A tensor may be its own result.  Its columns are neighbours in memory, its rows may have gaps between them.  What a call
    writes counts as changed in place; results take no part in autograd.
    bfloat16 results have an error of about their own rounding, 2e-3 of the norm (3e-3 where a matrix is a thousand times as long as wide); float32 and float16 results that of float32
    products, for three times the work.
    Work is enqueued on the stream the plan was made on (or `stream`); a call made while another stream is current orders the
    two.  One plan is for one stream and one host thread at a time.  Making one takes 0.5 to 1.5 ms (allocations, tables, a synchronisation): it is kept for a
    model, and outlives the graphs that captured its calls."""

    def __init__(self, shapes, dtypes=torch.float32, num_rows=1, steps=5, coefficients=COEFFICIENTS, eps=1e-7, result_dtypes=None,
                 device=None, stream=None):
        self.h, self._plan = None, _Closed()
        self.shapes = [tuple(int(n) for n in s) for s in shapes]
        if not self.shapes or any(len(s) < 2 for s in self.shapes):
            raise ValueError("shapes: at least one, each of two dimensions or more")
        self.K, self.T, self.steps = int(num_rows), len(self.shapes), int(steps)
        self.dtypes = _per_matrix(dtypes, self.T, "dtypes")
        self.result_dtypes = self.dtypes if result_dtypes is None else _per_matrix(result_dtypes, self.T, "result_dtypes")
        table = np.asarray(coefficients, dtype=np.float32)
        if table.shape == (3,):
            table = np.tile(table, (max(0, self.steps), 1))
        if table.shape != (self.steps, 3) or self.steps < 1:
            raise ValueError("coefficients: three numbers, or three for every one of at least one step")
        self.coefficients = np.ascontiguousarray(table)
        self.device = torch.device("cuda") if device is None else torch.device(device)
        if self.device.type != "cuda":
            raise ValueError("an orthogonaliser lives on a CUDA device")
        index = torch.cuda.current_device() if self.device.index is None else self.device.index
        self.device = torch.device("cuda", index)
        self.stream = torch.cuda.current_stream(self.device).cuda_stream if stream is None else int(stream)
        rows = np.array([s[0] for s in self.shapes], dtype=np.int64)
        cols = np.array([math.prod(s[1:]) for s in self.shapes], dtype=np.int64)
        types, results = (np.array([TYPE_OF[t] for t in kinds], dtype=np.int32) for kinds in (self.dtypes, self.result_dtypes))
        i64, i32, f32 = (C.POINTER(t) for t in (C.c_int64, C.c_int32, C.c_float))
        cfg = SaeOrthoConfig(ABI_VERSION, self.K, self.T, rows.ctypes.data_as(i64), cols.ctypes.data_as(i64), types.ctypes.data_as(i32),
                             results.ctypes.data_as(i32), self.steps, self.coefficients.ctypes.data_as(f32), eps, index, C.c_void_p(self.stream))
        h = C.c_void_p()
        self._check(binding.lib().sae_ortho_init(C.byref(cfg), C.byref(h)), "sae_ortho_init", None)
        self.h = h
        self._plan = binding.host().OrthoPlan(h.value, self.K, [list(s) for s in self.shapes], types.tolist(), results.tolist(), index, self.stream)

    @classmethod
    def like(cls, tensors, num_rows=1, **more):
        """The plan of tensors shaped like `tensors` (a model's matrices), of their dtypes."""
        tensors = list(tensors)
        if not tensors:
            raise ValueError("at least one tensor is wanted")
        return cls([t.shape for t in tensors], more.pop("dtypes", [t.dtype for t in tensors]), num_rows, device=more.pop("device", tensors[0].device), **more)

    @staticmethod
    def _check(status, what, h):
        if status != OK:
            raise SaeError(status, what, binding.lib().sae_ortho_last_cuda_error(h))

    def close(self):
        if self.h:
            self._plan = _Closed()
            binding.lib().sae_ortho_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __call__(self, tensors, results=None):
        status, results = self._plan.run(tensors, results)
        if status:
            self._check(status, "sae_ortho_run", self.h)
        return results
