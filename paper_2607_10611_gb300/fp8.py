"""Linear layers in 8 bits on torch tensors: E4M3 matrices with a power-of-two
scale per block of 128, their product, and a linear layer made of both, forward
and backward.  Argument marshalling around mpadam_e4m3_*, most of it in
csrc/torch_ext.cpp; no arithmetic here.

    x [tokens, k], w [n, k], dy [tokens, n]
    y  = q(x) q(w)^T         rows of x in blocks of 128 along k, w in squares
    dx = q(dy) q(w)          rows of dy along n, the same codes of w transposed
    dw = q(dy^T) q(x^T)^T    both transposes in blocks along the tokens
"""
from __future__ import annotations

from typing import Optional, Tuple, Union

import torch

from . import _native as N

BLOCK = 128
E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu


def scale_shape(rows: int, cols: int) -> Tuple[int, ...]:
    """Shape of a matrix's stored scales: [128-row tiles, groups of 4 blocks, 32, 4, 4]."""
    return (-(-rows // BLOCK), -(-cols // (4 * BLOCK)), 32, 4, 4)


class E4M3Matrix:
    """codes: float8_e4m3fn [rows, cols], row stride a multiple of 16; scales: float8_e8m0fnu of scale_shape(), as
    quantize() makes them."""

    __slots__ = ("codes", "scales")

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor):
        N.ext().check_matrix(codes, scales)
        self.codes, self.scales = codes, scales

    @property
    def shape(self):
        return self.codes.shape

    def row_scales(self) -> torch.Tensor:
        """Scales as float32 [rows, blocks of 128]."""
        rows, cols = self.codes.shape
        s = self.scales.float().permute(0, 3, 2, 1, 4).reshape(self.scales.shape[0] * BLOCK, self.scales.shape[1] * 4)
        return s[:rows, :-(-cols // BLOCK)]

    def dequantize(self) -> torch.Tensor:
        """The values the matrix stands for, float32 [rows, cols]."""
        return self.codes.float() * self.row_scales().repeat_interleave(BLOCK, 1)[:, :self.codes.shape[1]]


def _matrix(codes: torch.Tensor, scales: torch.Tensor) -> E4M3Matrix:
    m = object.__new__(E4M3Matrix)
    m.codes, m.scales = codes, scales
    return m


def quantize(x: torch.Tensor, *, square: bool = False, transposed: Union[bool, str] = False,
             stream: Optional[torch.cuda.Stream] = None):
    """x (CUDA float32 or bfloat16 [rows, cols] with contiguous rows) as an E4M3Matrix with a scale per 128 values of
    a row (square: per 128 x 128).  transposed: False: (x), True: the pair (x, its transpose), "only": the transpose
    alone; all from one pass over x."""
    if transposed not in (False, True, "only"):
        raise ValueError("transposed must be False, True or 'only'")
    if stream is not None:
        with torch.cuda.stream(stream):  # so that the results belong to it
            return quantize(x, square=square, transposed=transposed)
    q, s, qt, st = N.ext().quantize(x, square, transposed != "only", bool(transposed))
    if not transposed:
        return _matrix(q, s)
    return _matrix(qt, st) if transposed == "only" else (_matrix(q, s), _matrix(qt, st))


def matmul(a: E4M3Matrix, b: E4M3Matrix, *, out: Optional[torch.Tensor] = None,
           out_dtype: torch.dtype = torch.bfloat16, accumulate: bool = False,
           stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """a [m, k] times b [n, k] transposed: [m, n] of out_dtype (float32 or bfloat16), or into `out` (contiguous rows);
    accumulate: added to a float32 `out`."""
    if out_dtype not in (torch.float32, torch.bfloat16):
        raise ValueError("out_dtype must be float32 or bfloat16")
    if stream is not None:
        with torch.cuda.stream(stream):  # so that a new result belongs to it
            return matmul(a, b, out=out, out_dtype=out_dtype, accumulate=accumulate)
    return N.ext().matmul(a.codes, a.scales, b.codes, b.scales, out, out_dtype is torch.float32, accumulate)


def device_status(device=None, stream: Optional[torch.cuda.Stream] = None) -> int:
    """Waits for the stream; error bits of the products since the last call (0 = none): a bounded wait gave up."""
    dev = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)
    with torch.cuda.device(dev):
        return N.mpadam_e4m3_status((stream or torch.cuda.current_stream(dev)).cuda_stream)


def linear(x: torch.Tensor, w: Union[torch.Tensor, E4M3Matrix], *, grad_w: Optional[torch.Tensor] = None) -> torch.Tensor:
    """x [..., k] times w [n, k] transposed, in 8 bits, [..., n] of x's type (float32 or bfloat16), on the current
    stream.  w: float32 or bfloat16, quantised in squares here, or (for serving, without gradients) an E4M3Matrix that
    quantize(w, square=True) made once.  Differentiable once in x and w, backwards only; grad_w: a float32 [n, k] to which a
    backward pass that asks for w's gradient adds it instead of returning it."""
    if isinstance(w, E4M3Matrix):
        if grad_w is not None:
            raise ValueError("a quantised weight passes no gradient")
        return N.ext().linear_held(x, w.codes, w.scales)
    return N.ext().linear(x, w, grad_w)
