"""Linear layers in 8 bits on torch tensors: E4M3 matrices with a power-of-two
scale per block of 128, their product, and a linear layer made of both, forward
and backward (argument marshalling around mpadam_e4m3_*; no arithmetic here).

    x [tokens, k], w [n, k], dy [tokens, n]
    y  = q(x) q(w)^T         rows of x in blocks of 128 along k, w in squares
    dx = q(dy) q(w)          rows of dy along n, the same codes of w transposed
    dw = q(dy^T) q(x^T)^T    both transposes in blocks along the tokens
"""
from __future__ import annotations

from typing import Optional, Tuple, Union

import torch

from . import _native as N
from .optimizer import _raw_stream

BLOCK = 128
E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu
_DTYPE = {torch.float32: N.MPADAM_F32, torch.bfloat16: N.MPADAM_BF16}


def scale_shape(rows: int, cols: int) -> Tuple[int, ...]:
    """Shape of a matrix's stored scales: [128-row tiles, groups of 4 blocks, 32, 4, 4]."""
    return (-(-rows // BLOCK), -(-cols // (4 * BLOCK)), 32, 4, 4)


class E4M3Matrix:
    """codes: float8_e4m3fn [rows, cols], row stride a multiple of 16; scales: float8_e8m0fnu of scale_shape(), as
    quantize() makes them."""

    __slots__ = ("codes", "scales")

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor):
        if codes.dtype != E4M3 or codes.dim() != 2 or not codes.is_cuda:
            raise ValueError("codes must be a CUDA float8_e4m3fn matrix")
        rows, cols = codes.shape
        if cols and rows and ((cols > 1 and codes.stride(1) != 1) or (rows > 1 and codes.stride(0) < cols)):
            raise ValueError("codes must have contiguous rows")
        if scales.dtype != E8M0 or tuple(scales.shape) != scale_shape(rows, cols) or not scales.is_contiguous() \
                or scales.device != codes.device:
            raise ValueError(f"scales must be a contiguous float8_e8m0fnu tensor of {scale_shape(rows, cols)} beside "
                             "the codes")
        self.codes, self.scales = codes, scales

    @classmethod
    def empty(cls, rows: int, cols: int, device) -> "E4M3Matrix":
        store = torch.empty(rows, -(-cols // 16) * 16, dtype=E4M3, device=device)
        return cls(store[:, :cols], torch.empty(scale_shape(rows, cols), dtype=E8M0, device=device))

    @property
    def shape(self):
        return self.codes.shape

    def row_scales(self) -> torch.Tensor:
        """Scales as float32 [rows, blocks of 128]."""
        rows, cols = self.codes.shape
        s = self.scales.float().permute(0, 3, 2, 1, 4).reshape(self.scales.shape[0] * BLOCK, -1)
        return s[:rows, :-(-cols // BLOCK)]

    def dequantize(self) -> torch.Tensor:
        """The values the matrix stands for, float32 [rows, cols]."""
        return self.codes.float() * self.row_scales().repeat_interleave(BLOCK, 1)[:, :self.codes.shape[1]]

    def _operand(self):
        """(codes, scales, row stride); a single row's stride is of no matter, so its codes may have any."""
        rows, cols = self.codes.shape
        ld = self.codes.stride(0) if rows > 1 else -(-cols // 16) * 16
        return self.codes.data_ptr(), self.scales.data_ptr(), ld


def quantize(x: torch.Tensor, *, square: bool = False, transposed: Union[bool, str] = False,
             stream: Optional[torch.cuda.Stream] = None):
    """x (CUDA float32 or bfloat16 [rows, cols] with contiguous rows) as an E4M3Matrix with a scale per 128 values of
    a row (square: per 128 x 128).  transposed: False: (x), True: the pair (x, its transpose), "only": the transpose
    alone; all from one pass over x."""
    if x.dim() != 2 or x.dtype not in _DTYPE or not x.is_cuda:
        raise ValueError("x must be a CUDA float32 or bfloat16 matrix")
    rows, cols = x.shape
    if rows and cols and ((cols > 1 and x.stride(1) != 1) or (rows > 1 and x.stride(0) < cols)):
        raise ValueError("x must have contiguous rows")
    if transposed not in (False, True, "only"):
        raise ValueError("transposed must be False, True or 'only'")
    q = E4M3Matrix.empty(rows, cols, x.device) if transposed != "only" else None
    qt = E4M3Matrix.empty(cols, rows, x.device) if transposed else None
    a = q._operand() if q else (0, 0, 0)
    b = qt._operand() if qt else (0, 0, 0)
    s = stream.cuda_stream if stream else _raw_stream(x.device)
    with torch.cuda.device(x.device):
        N.mpadam_e4m3_quantize(x.data_ptr(), _DTYPE[x.dtype], rows, cols, max(x.stride(0), cols) if rows > 1 else cols,
                               int(square), *a, *b, s)
    return q if not transposed else qt if transposed == "only" else (q, qt)


def matmul(a: E4M3Matrix, b: E4M3Matrix, *, out: Optional[torch.Tensor] = None,
           out_dtype: torch.dtype = torch.bfloat16, accumulate: bool = False,
           stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """a [m, k] times b [n, k] transposed: [m, n] of out_dtype (float32 or bfloat16), or into `out` (contiguous rows);
    accumulate: added to a float32 `out`."""
    (m, k), (n, kb) = a.shape, b.shape
    if k != kb:
        raise ValueError(f"inner sizes differ: {k} and {kb}")
    dev = a.codes.device
    if out is None:
        if accumulate:
            raise ValueError("accumulate needs out")
        out = torch.empty(m, n, dtype=out_dtype, device=dev)
    if out.dtype not in _DTYPE or tuple(out.shape) != (m, n) or out.device != dev or b.codes.device != dev or \
            (m and n and ((n > 1 and out.stride(1) != 1) or (m > 1 and out.stride(0) < n))):
        raise ValueError(f"out must be a float32 or bfloat16 [{m}, {n}] with contiguous rows beside the operands")
    p = N.mpadam_e4m3_product(*a._operand(), *b._operand(), out.data_ptr(), max(out.stride(0), n) if m > 1 else n,
                              m, n, k, _DTYPE[out.dtype], int(accumulate))
    s = stream.cuda_stream if stream else _raw_stream(dev)
    with torch.cuda.device(dev):
        N.mpadam_e4m3_matmul(p, s)
    return out


def device_status(device=None, stream: Optional[torch.cuda.Stream] = None) -> int:
    """Waits for the stream; error bits of the products since the last call (0 = none): a bounded wait gave up."""
    dev = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)
    with torch.cuda.device(dev):
        return N.mpadam_e4m3_status((stream or torch.cuda.current_stream(dev)).cuda_stream)


def _rows(x: torch.Tensor) -> torch.Tensor:
    """x as a matrix of its last dimension, with contiguous rows."""
    x = x.reshape(-1, x.shape[-1])
    return x if x.shape[1] <= 1 or (x.stride(1) == 1 and (x.shape[0] <= 1 or x.stride(0) >= x.shape[1])) \
        else x.contiguous()


class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, grad_w):
        rows = _rows(x.detach())
        need_x, need_w = ctx.needs_input_grad[:2]
        q, qt = quantize(rows, transposed=True) if need_w else (quantize(rows), None)
        if isinstance(w, E4M3Matrix):
            qw, qwt = w, None
        elif need_x:
            qw, qwt = quantize(_rows(w.detach()), square=True, transposed=True)
        else:
            qw, qwt = quantize(_rows(w.detach()), square=True), None
        ctx.qt, ctx.qwt, ctx.grad_w = qt, qwt, grad_w
        ctx.x_shape, ctx.w_dtype, ctx.x_dtype = x.shape, None if isinstance(w, E4M3Matrix) else w.dtype, x.dtype
        return matmul(q, qw, out_dtype=x.dtype).view(*x.shape[:-1], qw.shape[0])

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        rows = _rows(dy)
        need_x, need_w = ctx.needs_input_grad[:2]
        if need_x and need_w:
            q, qt = quantize(rows, transposed=True)
        else:
            q, qt = (quantize(rows), None) if need_x else (None, quantize(rows, transposed="only"))
        dx = matmul(q, ctx.qwt, out_dtype=ctx.x_dtype).view(ctx.x_shape) if need_x else None
        dw = None
        if need_w:
            if ctx.grad_w is not None:
                matmul(qt, ctx.qt, out=ctx.grad_w, accumulate=True)
            else:
                dw = matmul(qt, ctx.qt, out_dtype=ctx.w_dtype)
        return dx, dw, None


def linear(x: torch.Tensor, w: Union[torch.Tensor, E4M3Matrix], *, grad_w: Optional[torch.Tensor] = None) -> torch.Tensor:
    """x [..., k] times w [n, k] transposed, in 8 bits, [..., n] of x's type (float32 or bfloat16), on the current
    stream.  w: float32 or bfloat16, quantised in squares here, or (for serving, without gradients) an E4M3Matrix that
    quantize(w, square=True) made once.  Differentiable once in x and w; grad_w: a float32 [n, k] to which the
    backward pass adds w's gradient instead of returning it."""
    if x.dim() < 1 or x.dtype not in _DTYPE or not x.is_cuda:
        raise ValueError("x must be a CUDA float32 or bfloat16 tensor")
    quantised = isinstance(w, E4M3Matrix)
    if not quantised and (w.dim() != 2 or w.dtype not in _DTYPE or w.device != x.device):
        raise ValueError("w must be a float32 or bfloat16 matrix beside x")
    if w.shape[1] != x.shape[-1]:
        raise ValueError(f"inner sizes differ: {x.shape[-1]} and {w.shape[1]}")
    if grad_w is not None and (grad_w.dtype != torch.float32 or tuple(grad_w.shape) != tuple(w.shape)
                               or grad_w.device != x.device or quantised):
        raise ValueError("grad_w must be a float32 tensor of w's shape beside it")
    if quantised:
        if x.requires_grad and torch.is_grad_enabled():
            raise ValueError("a quantised weight passes no gradient: give linear() the weight itself")
        return matmul(quantize(_rows(x)), w, out_dtype=x.dtype).view(*x.shape[:-1], w.shape[0])
    return _Linear.apply(x, w, grad_w)
