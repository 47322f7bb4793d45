"""GB300-native fused M+Adam optimizer step (arxiv 2607.10611), and what trains
a layer next to it: AdamW with moments in binary32 or 8 bits, Muon and the
orthogonalisation it is made of, the gradients' norm, block-of-128 E4M3
matrices, their product and a linear layer, layer normalisation, and products
with NVFP4 weights.

The kernels are hand-written for sm_103a behind the C ABI of include/mpadam.h;
this package holds that library's sources (csrc/), its build script, a thin
ctypes binding with the C entry points' names and classes on torch tensors
(MPAdam, AdamW, Muon, Orthogonalizer, GradNorm, layer_norm, fp8, fp4).  PyTorch is used for device memory, streams and
the layers' place in the graph.
"""
from .builder import build  # noqa: F401

__all__ = ["build", "native", "MPAdam", "AdamW", "GradNorm", "Muon", "Orthogonalizer", "fp8", "fp4", "layer_norm"]


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
    if name in ("Muon", "Orthogonalizer"):
        from . import muon
        return getattr(muon, name)
    if name in ("fp8", "fp4"):
        import importlib
        return importlib.import_module("." + name, __name__)
    if name == "layer_norm":
        from .norm import layer_norm
        return layer_norm
    raise AttributeError(name)
