"""Dense operators beside the binary network (include/bmlp.h has the formulas):
root-mean-square norm with the residual's addition and int8 rows with a scale
each, its gradient, the product of such rows with 8-bit weights, and the
distillation loss against a teacher's top logits with its gradient.

Everything is computed by the HIP library on the current torch stream of the
tensors' device, and nothing here waits for it.  The calls on tensors (argument
checks, output allocation, the C entries) are compiled, in
binding/dense_binding.cpp; if that module or the library has not been built,
importing this one raises.  Matrices may be rows cut out of wider ones (a row
stride); the elements of a row are contiguous.  Arguments that do not fit raise
ValueError, a status of the library BmlpError.

Nothing here is recorded for autograd.  A tensor that requires a gradient is
refused while gradients are recorded: pass it detached and chain the gradients
that ``norm_quant_backward`` and ``distill`` return, for example
``logits.backward(distill(logits.detach(), ...)[1])``.
"""
from __future__ import annotations

import importlib.util
import os
from typing import NamedTuple, Optional

import torch

from .bmlp import BmlpError, _raw_stream_getter, lib
from .build import BINDING_PATH


def _load_binding():
    lib()   # raises if the library is missing
    if not os.path.exists(BINDING_PATH):
        raise RuntimeError(f"extension module {BINDING_PATH} is missing; build it with "
                           "paper_2412_00119_amd.build.build()")
    spec = importlib.util.spec_from_file_location("_dense_binding", BINDING_PATH)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)

    def fail(status, name):
        raise BmlpError(status, name)

    mod.bind(_raw_stream_getter(torch), fail)
    return mod


_c = _load_binding()
TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}   # BMLP_TYPE_*


class NormQuant(NamedTuple):
    q: torch.Tensor                  # int8 [n][K]
    scale: torch.Tensor              # float32 [n]
    rstd: torch.Tensor               # float32 [n]
    h: Optional[torch.Tensor]        # x + residual, in x's type (None without a residual: h is x)
    y: Optional[torch.Tensor]        # q * scale, in x's type


_new = tuple.__new__


def norm_quant(x, weight=None, residual=None, eps: float = 1e-6, values: bool = False) -> NormQuant:
    """Root-mean-square norm of x + residual as int8 rows with a scale each.

    ``values`` also returns the values that the rows stand for, in x's type.
    The rows are contiguous, as ``expand``, ``feature_median`` and ``binarize``
    take them."""
    return _new(NormQuant, _c.norm_quant(x, weight, residual, eps, values))


def quantize_rows(x):
    """int8 rows and their scales (largest |x| over 127): (q [n][K], scale [n])."""
    return _c.quantize_rows(x)


def norm_quant_backward(dy, h, rstd, weight=None, dh=None):
    """Gradient of ``norm_quant`` straight through the rounding: (dx, dweight).

    dy is the gradient of y, h and rstd are the forward call's (h is x where it
    had no residual), dh the gradient that reaches h along the residual path.
    dx is the gradient of x and of the residual alike; dweight is None without
    a weight."""
    return _c.norm_quant_backward(dy, h, rstd, weight, dh)


class QLinear:
    """A layer of 8-bit weights [N][K] with a scale for each of the N outputs.

    The weights are laid out for the matrix cores once, here; w itself is not
    kept.  Inference only: the layer is made of constants, from parameters too."""

    def __init__(self, w, scale, bias=None):
        with torch.no_grad():
            self.packed, = _c.qlinear_pack(w, scale, bias)
        self.n_out, self.n_in = w.shape
        self.scale, self.bias = scale.detach(), None if bias is None else bias.detach()

    @classmethod
    def from_weight(cls, w, bias=None):
        """From real-valued weights [N][K], quantised row by row."""
        with torch.no_grad():
            return cls(*quantize_rows(w), bias)

    def __call__(self, q, scale=None, dtype=torch.bfloat16):
        """q int8 [n][K] with a scale for each row (None: ones) -> [n][N] of dtype."""
        return _c.qlinear(q, scale, dtype, self.packed, self.scale, self.bias, self.n_in, self.n_out)


def distill(z, idx, t, tau: float = 1.0, lse=None, weight=None, grad: bool = True):
    """Distillation of the logits z [n][c] from a teacher's listed classes idx
    (int32 [n][k], -1: no entry) with logits t [n][k] at temperature tau:
    (loss float32 [n], gradient of the weighted losses' sum in z's type or None).

    lse float32 [n], if given, is the logarithm of the sum of exp(t / tau) over
    all of the teacher's classes: those it did not list then count as one more
    outcome.  weight float32 [n] multiplies each row's loss and gradient."""
    return _c.distill(z, idx, t, tau, lse, weight, grad)
