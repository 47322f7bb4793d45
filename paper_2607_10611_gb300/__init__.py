"""GB300-native fused M+Adam optimizer step (arxiv 2607.10611), and what trains
a layer in 8 bits next to it: AdamW with moments in binary32 or 8 bits, the
gradients' norm, block-of-128 E4M3 matrices, their product and a linear layer.

The kernels are hand-written for sm_103a behind the C ABI of include/mpadam.h;
this package holds that library's sources (csrc/), its build script, a thin
ctypes binding with the C entry points' names and classes on torch tensors
(MPAdam, AdamW, GradNorm, fp8).  PyTorch is used for device memory, streams and
the layer's place in the graph.
"""
from .builder import build  # noqa: F401

__all__ = ["build", "native", "MPAdam", "AdamW", "GradNorm", "fp8"]


def __getattr__(name):
    if name == "native":
        from . import _native
        return _native
    if name == "MPAdam":
        from .optimizer import MPAdam
        return MPAdam
    if name in ("AdamW", "GradNorm"):
        from . import adamw
        return getattr(adamw, name)
    if name == "fp8":
        import importlib
        return importlib.import_module(".fp8", __name__)
    raise AttributeError(name)
