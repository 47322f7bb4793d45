"""Muon and the orthogonalisation it is made of over lists of torch matrices:
argument marshalling around mpadam_muon_* and mpadam_orthogonal_* (no arithmetic
here).  What every call does with its list is csrc/torch_ext.cpp's.
"""
from __future__ import annotations

import ctypes
from typing import List, Optional, Sequence, Tuple

import torch

from . import _native as N

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


class Orthogonalizer:
    """Matrices of the given shapes, float32 or bfloat16, each by `steps` Newton-Schulz steps nearly its polar factor: its
    singular values come to lie around 1, its singular vectors stay.  Products are of FP16 values, so that a result, float32 or
    bfloat16, is good to about 1.4e-3 of itself (2-norm).  The workspace is the object's, so calls on several streams have to be
    ordered."""

    def __init__(self, shapes: Sequence[Tuple[int, int]], dtype: str = "bf16", steps: int = 5,
                 device: Optional[torch.device] = None):
        self.shapes = [(int(r), int(c)) for r, c in shapes]
        device = torch.device("cuda" if device is None else device)
        if device.index is None:
            device = torch.device("cuda", torch.cuda.current_device())
        self.device = device
        with torch.cuda.device(device):
            self.state = N.mpadam_orthogonal_create(self.shapes, N.DTYPE[dtype], steps)
        self._spec = N.ext().matrix_spec(self.shapes, dtype == "f32", device.index)
        self._run = N.ext().orthogonalize

    def __call__(self, x: Sequence[torch.Tensor], out: Optional[Sequence[torch.Tensor]] = None,
                 stream: Optional[torch.cuda.Stream] = None) -> List[torch.Tensor]:
        """The orthogonalised matrices, asynchronously: new ones, or written to `out` (entries may be x's own, but none another's)."""
        if stream is None:
            return self._run(self.state, self._spec, x, out, None)
        with torch.cuda.stream(stream):  # so that new results belong to it
            return self._run(self.state, self._spec, x, out, None)

    def device_status(self) -> int:
        """Device error bits of the calls so far (0 = none); synchronises."""
        with torch.cuda.device(self.device):
            return N.mpadam_orthogonal_status(self.state)

    def close(self):
        if getattr(self, "state", None):
            with torch.cuda.device(self.device):
                N.mpadam_orthogonal_destroy(self.state)
            self.state = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Muon:
    """One Muon step per call over every matrix of a list.

    w: contiguous CUDA matrices of `weight_dtype` ("f32" or "bf16"), updated in
    place, as is the momentum m, matrices of the same shapes of `momentum_dtype`
    ("f32" or "bf16"); init_state() makes it.  scale: what the learning rate of a
    matrix is multiplied by, "rms" (0.2 sqrt of its longer side) or "spectral"
    (sqrt of rows / columns, at least 1).  rounding is that of BF16 weights
    (binary32 ones need none).  compute: with binary32 weights, BF16 matrices that
    every step overwrites with the rounded weights (entries may be None).  The
    tensors' memory has to stay where it is; the object keeps references to them,
    and a workspace, so calls on several streams have to be ordered.  An update is
    good to about 1.4e-3 of itself, as Orthogonalizer's results are.  Vectors,
    embeddings and the head are AdamW's.
    """

    def __init__(self, w: Sequence[torch.Tensor], m: Sequence[torch.Tensor], *,
                 compute: Optional[Sequence[Optional[torch.Tensor]]] = None, weight_dtype: str = "bf16",
                 grad_dtype: str = "bf16", momentum_dtype: str = "f32", rounding: str = "nearest", seed: int = 0,
                 momentum: float = 0.95, nesterov: bool = True, weight_decay: float = 0.01, steps: int = 5,
                 scale: str = "rms"):
        self.w, self.m = list(w), list(m)
        self.compute = list(compute) if compute is not None else None
        cfg = N.mpadam_muon_config(momentum, weight_decay, int(nesterov), steps, N.MUON_SCALES[scale], N.DTYPE[weight_dtype],
                                   N.DTYPE[grad_dtype], N.DTYPE[momentum_dtype], N.ROUNDING[rounding], 0, seed)
        self.state = N.ext().muon_create(ctypes.addressof(cfg), self.w, self.m, self.compute)
        self.device = self.w[0].device if self.w else torch.device("cuda", torch.cuda.current_device())
        self._spec = N.ext().matrix_spec([tuple(t.shape) for t in self.w], grad_dtype == "f32", self.device.index)
        self._step = N.ext().muon_step

    @staticmethod
    def init_state(w: Sequence[torch.Tensor], momentum_dtype: str = "f32") -> dict:
        """Zero momentum for the weights w, as keyword arguments of Muon: m, momentum_dtype."""
        return {"m": [torch.zeros(t.shape, dtype=_TYPES[momentum_dtype], device=t.device) for t in w],
                "momentum_dtype": momentum_dtype}

    def step(self, grads: Sequence[torch.Tensor], t: int, lr: float, grad_scale: Optional[torch.Tensor] = None,
             stream: Optional[torch.cuda.Stream] = None):
        """Step t (from 1) with learning rate lr, asynchronously.  grad_scale: a CUDA float32 tensor whose first
        element multiplies every gradient (GradNorm's [1:]), NaN: the step changes nothing."""
        self._step(self.state, self._spec, grads, t, lr, grad_scale, stream.cuda_stream if stream else None)

    def device_status(self) -> int:
        """Device error bits of the steps so far (0 = none); synchronises.  While they are not 0, steps leave weights alone."""
        with torch.cuda.device(self.device):
            return N.mpadam_muon_status(self.state)

    def close(self):
        if getattr(self, "state", None):
            with torch.cuda.device(self.device):
                N.mpadam_muon_destroy(self.state)
            self.state = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
