"""AdamW and the global gradient norm over lists of torch tensors: argument
marshalling around mpadam_adamw_* and mpadam_grad_norm_* (no arithmetic here).
What every call does with its list of gradients is csrc/torch_ext.cpp's.
"""
from __future__ import annotations

import ctypes
from typing import Optional, Sequence

import torch

from . import _native as N

_STATE = {"f32": torch.float32, "e4m3": torch.float8_e4m3fn}
BLOCK = 128  # elements that share a scale of 8-bit moments


class AdamW:
    """One fused AdamW step per call over every tensor of a list.

    w: contiguous CUDA tensors of `weight_dtype` ("f32" or "bf16"), updated in
    place, as are the moments m and v: binary32 tensors (state_dtype "f32"), or
    (state_dtype "e4m3") float8_e4m3fn tensors of the same sizes with m_scales
    and v_scales, float8_e8m0fnu tensors of ceil(numel / 128) scales each; v then
    holds the second moment's square root.  init_state() makes either.
    rounding is that of BF16 weights (binary32 ones need none).
    compute: with binary32 weights, BF16 tensors that every step overwrites with
    the rounded weights (entries may be None).  The tensors' memory has to stay
    where it is; the object keeps references to them.
    """

    def __init__(self, w: Sequence[torch.Tensor], m: Sequence[torch.Tensor], v: Sequence[torch.Tensor], *,
                 m_scales: Optional[Sequence[torch.Tensor]] = None,
                 v_scales: Optional[Sequence[torch.Tensor]] = None,
                 compute: Optional[Sequence[Optional[torch.Tensor]]] = None, weight_dtype: str = "bf16",
                 grad_dtype: str = "bf16", state_dtype: str = "f32", rounding: str = "nearest",
                 state_rounding: Optional[str] = None, seed: int = 0, beta1: float = 0.9, beta2: float = 0.999,
                 eps: float = 1e-8, weight_decay: float = 0.01):
        self.w, self.m, self.v = list(w), list(m), list(v)
        given = lambda x: list(x) if x is not None else None
        self.m_scales, self.v_scales, self.compute = given(m_scales), given(v_scales), given(compute)
        if state_rounding is None:
            state_rounding = "stochastic" if state_dtype == "e4m3" else "nearest"
        cfg = N.mpadam_adamw_config(beta1, beta2, eps, weight_decay, N.DTYPE[weight_dtype], N.DTYPE[grad_dtype],
                                    N.DTYPE[state_dtype], N.ROUNDING[rounding], N.ROUNDING[state_rounding], 0, seed)
        self.state = N.ext().adamw_create(ctypes.addressof(cfg), self.w, self.m, self.v, self.m_scales, self.v_scales,
                                          self.compute)
        self.device = self.w[0].device if self.w else torch.device("cuda", torch.cuda.current_device())
        self.numels = [t.numel() for t in self.w]
        self._spec = N.ext().list_spec(self.numels, grad_dtype == "f32", self.device.index)
        self._step = N.ext().adamw_step

    @staticmethod
    def init_state(w: Sequence[torch.Tensor], state_dtype: str = "e4m3") -> dict:
        """Zero moments for the weights w, as keyword arguments of AdamW: m, v (and m_scales, v_scales)."""
        new = lambda: [torch.zeros(t.shape, dtype=_STATE[state_dtype], device=t.device) for t in w]
        got = {"m": new(), "v": new(), "state_dtype": state_dtype}
        if state_dtype == "e4m3":
            one = lambda t: torch.full((-(-t.numel() // BLOCK),), 127, dtype=torch.uint8,
                                       device=t.device).view(torch.float8_e8m0fnu)
            got.update(m_scales=[one(t) for t in w], v_scales=[one(t) for t in w])
        return got

    def step(self, grads: Sequence[torch.Tensor], t: int, lr: float, grad_scale: Optional[torch.Tensor] = None,
             stream: Optional[torch.cuda.Stream] = None):
        """Step t (from 1) with learning rate lr, asynchronously.  grad_scale: a CUDA float32 tensor whose first
        element multiplies every gradient (GradNorm's [1:]), NaN: the step changes nothing."""
        self._step(self.state, self._spec, grads, t, lr, grad_scale, stream.cuda_stream if stream else None)

    def device_status(self) -> int:
        """Device error bits of the steps so far (0 = none); synchronises."""
        with torch.cuda.device(self.device):
            return N.mpadam_adamw_status(self.state)

    def close(self):
        if getattr(self, "state", None):
            with torch.cuda.device(self.device):
                N.mpadam_adamw_destroy(self.state)
            self.state = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class GradNorm:
    """The global 2-norm of a list of gradients with the given sizes, and the multiplier that clips them.  Its partial
    sums are the object's, so calls on several streams have to be ordered, as AdamW's have to be."""

    def __init__(self, numels: Sequence[int], grad_dtype: str = "bf16", device: Optional[torch.device] = None):
        self.numels = [int(n) for n in numels]
        device = torch.device("cuda" if device is None else device)
        if device.index is None:
            device = torch.device("cuda", torch.cuda.current_device())
        self.device = device
        with torch.cuda.device(device):
            self.state = N.mpadam_grad_norm_create(self.numels, N.DTYPE[grad_dtype])
        self._spec = N.ext().list_spec(self.numels, grad_dtype == "f32", device.index)
        self._norm = N.ext().grad_norm

    def __call__(self, grads: Sequence[torch.Tensor], max_norm: float = float("inf"),
                 out: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
        """float32 [2], asynchronously: the norm, and min(1, max_norm / norm) (NaN when the norm is not finite)."""
        if stream is None:
            return self._norm(self.state, self._spec, grads, max_norm, out, None)
        with torch.cuda.stream(stream):  # so that a new out belongs to it
            return self._norm(self.state, self._spec, grads, max_norm, out, None)

    def close(self):
        if getattr(self, "state", None):
            with torch.cuda.device(self.device):
                N.mpadam_grad_norm_destroy(self.state)
            self.state = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
