"""Weights in NVFP4 as M+Adam's step leaves them (MPAdam with weight_dtype
"nvfp4"), times few tokens: what serves a layer that was trained so, without
another copy of its weight.  Argument marshalling around mpadam_nvfp4_linear,
in csrc/torch_ext.cpp; no arithmetic here.
"""
from __future__ import annotations

from typing import Tuple

import torch

from . import _native as N

GROUP = 16  # consecutive elements of the flat weight that share a scale


class NVFP4Matrix:
    """A weight of `shape` (rows, columns): codes, uint8, two E2M1 codes a byte, the first in the low nibble; scales, E4M3
    codes (uint8 or float8_e4m3fn), one per 16 consecutive elements of the flat weight; global_scale, the tensor's.  The
    tensors are those that MPAdam holds, of any shape; they are kept, not copied, so a step changes the matrix too."""

    __slots__ = ("codes", "scales", "global_scale", "shape")

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor, global_scale: float, shape: Tuple[int, int]):
        rows, cols = (int(n) for n in shape)
        N.ext().check_nvfp4(codes, scales, global_scale, rows, cols)
        self.codes, self.scales, self.global_scale, self.shape = codes, scales, float(global_scale), torch.Size((rows, cols))

    def dequantize(self) -> torch.Tensor:
        """The values the matrix stands for, float32 [rows, columns]."""
        n = self.shape.numel()
        pairs = self.codes.reshape(-1)
        codes = torch.stack([pairs & 15, pairs >> 4], 1).view(-1)[:n].long()
        values = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], device=codes.device)[codes]
        scales = self.scales.reshape(-1).view(torch.float8_e4m3fn).float() * self.global_scale
        return (values * scales.repeat_interleave(GROUP)[:n]).view(self.shape)


def linear(x: torch.Tensor, w: NVFP4Matrix) -> torch.Tensor:
    """x [..., k] (CUDA float32 or bfloat16) times w [n, k] transposed, [..., n] of x's type, on the current stream, without
    gradients.  Products are exact, sums in binary32.  Made for a token or a few: w is read once for every 8 to 32 rows of x
    (fp8.linear with a held weight takes more)."""
    return N.ext().nvfp4_linear(x, w.codes, w.scales, w.global_scale, *w.shape)
