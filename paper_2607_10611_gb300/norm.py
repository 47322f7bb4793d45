"""Layer normalisation on torch tensors: argument marshalling around
mpadam_layer_norm_*, in csrc/torch_ext.cpp; no arithmetic here.
"""
from __future__ import annotations

from typing import Optional

import torch

from . import _native as N


def layer_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, *,
               eps: float = 1e-5) -> torch.Tensor:
    """x [..., d] (CUDA float32 or bfloat16) normalised over its last dimension, times weight, plus bias (d elements each,
    float32 or of x's type, or None), of x's type, on the current stream.  Statistics and sums are in binary32.
    Differentiable once in x, weight and bias, backwards only; the gradients have their tensors' types, and the same call
    gives the same bits."""
    return N.ext().layer_norm(x, weight, bias, eps)
