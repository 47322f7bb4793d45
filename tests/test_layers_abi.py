"""Refusals of the layer norm's and the NVFP4 product's entry points that are decided on the host, before any CUDA call (no
GPU needed)."""
import math

import pytest

from paper_2607_10611_gb300 import builder as B


@pytest.fixture(scope="module")
def N():
    B.build()
    from paper_2607_10611_gb300 import _native
    return _native


def refused(N, f, *args, **kw):
    with pytest.raises(N.MPAdamError) as ei:
        f(*args, **kw)
    assert ei.value.status == N.MPADAM_EINVAL and N.mpadam_last_error()


FORWARD = dict(x=0x1000, ldx=20, w=0x2000, b=0x3000, y=0x4000, ldy=24, mean=0x5000, rstd=0x6000, rows=5, cols=20, x_dtype=1,
               w_dtype=0, eps=1e-5, reserved=0)
BACKWARD = dict(x=0x1000, ldx=20, dy=0x2000, lddy=20, w=0x3000, mean=0x4000, rstd=0x5000, dx=0x6000, lddx=20, dw=0x7000,
                db=0x8000, workspace=0x9000, workspace_bytes=1 << 30, rows=5, cols=20, x_dtype=1, w_dtype=0)
BOTH = [dict(rows=-1), dict(cols=-1), dict(rows=1 << 31), dict(cols=1 << 31), dict(x_dtype=2), dict(x_dtype=-1), dict(w_dtype=2),
        dict(x_dtype=0, w_dtype=1), dict(x=None), dict(x=0x1001), dict(ldx=19), dict(w=0x2002), dict(mean=0x5002),
        dict(rstd=0x6001), dict(mean=None)]


@pytest.mark.parametrize("bad", BOTH + [dict(b=0x3001), dict(y=None), dict(y=0x4001), dict(ldy=19), dict(eps=-1e-9),
                                        dict(eps=math.nan), dict(eps=math.inf), dict(reserved=1)])
def test_the_norms_forward_pass_refuses(N, bad):
    refused(N, N.mpadam_layer_norm_forward, N.mpadam_layer_norm(**{**FORWARD, **bad}))


@pytest.mark.parametrize("bad", BOTH + [dict(dy=None), dict(dy=0x2001), dict(lddy=19), dict(dx=0x6001), dict(lddx=19),
                                        dict(dw=0x7002), dict(db=0x8001), dict(rstd=None), dict(workspace=None),
                                        dict(workspace=0x9008), dict(workspace_bytes=2 * 20 * 4 - 1)])
def test_the_norms_backward_pass_refuses(N, bad):
    refused(N, N.mpadam_layer_norm_backward, N.mpadam_layer_norm_grad(**{**BACKWARD, **bad}))


def test_norms_of_nothing_need_no_pointers(N):
    nothing = dict(x=None, w=None, b=None, y=None, mean=None, rstd=None)
    for sizes in (dict(rows=0), dict(cols=0)):
        N.mpadam_layer_norm_forward(N.mpadam_layer_norm(**{**FORWARD, **nothing, **sizes}))
    none = dict(x=None, dy=None, dx=None, dw=None, db=None, mean=None, rstd=None, workspace=None, workspace_bytes=0)
    for sizes in (dict(rows=0), dict(cols=0), {}):  # without rows nothing is cleared where nothing is wanted
        N.mpadam_layer_norm_backward(N.mpadam_layer_norm_grad(**{**BACKWARD, **none, **sizes}))


def test_the_norms_workspace(N):
    for rows, cols in ((-1, 1), (1, -1), (1 << 31, 1), (1, 1 << 31)):
        refused(N, N.mpadam_layer_norm_workspace, rows, cols)
    assert N.mpadam_layer_norm_workspace(0, 5) == N.mpadam_layer_norm_workspace(5, 0) == 0
    top = (1 << 31) - 1
    for rows in (1, 7, 8, 9, 1000, 1 << 20, top):
        for cols in (1, 768, 1024, 1025, 8192, 8193, 1 << 20, top):
            parts, rest = divmod(N.mpadam_layer_norm_workspace(rows, cols), 8 * cols)
            assert rest == 0 and 1 <= parts <= min(rows, 608)


WEIGHT = dict(codes=0x10000, scales=0x20000, rows=7, cols=64, global_scale=0.5, reserved=0)
CALL = dict(x=0x1000, x_dtype=1, tokens=3, ldx=64, y=0x30000, ldy=7)


@pytest.mark.parametrize("bad", [
    dict(rows=-1), dict(cols=-1), dict(rows=1 << 31), dict(cols=1 << 31), dict(global_scale=0.0), dict(global_scale=-1.0),
    dict(global_scale=math.nan), dict(global_scale=math.inf), dict(reserved=1), dict(codes=None), dict(scales=None), dict(x=0),
    dict(x=0x1001), dict(x_dtype=2), dict(tokens=-1), dict(tokens=(1 << 16) + 1), dict(ldx=63), dict(y=0), dict(y=0x30001),
    dict(ldy=6)])
def test_the_nvfp4_product_refuses(N, bad):
    weight = N.mpadam_nvfp4_matrix(**{**WEIGHT, **{k: v for k, v in bad.items() if k in WEIGHT}})
    refused(N, N.mpadam_nvfp4_linear, **{**CALL, **{k: v for k, v in bad.items() if k in CALL}}, w=weight)


def test_nvfp4_products_of_nothing_need_no_pointers(N):
    none = dict(x=0, y=0)
    N.mpadam_nvfp4_linear(**{**CALL, **none, "tokens": 0}, w=N.mpadam_nvfp4_matrix(**WEIGHT))
    N.mpadam_nvfp4_linear(**{**CALL, **none}, w=N.mpadam_nvfp4_matrix(**{**WEIGHT, "rows": 0, "codes": None, "scales": None}))


def test_tensors_that_no_layer_takes_are_refused(N):
    """By the torch side, on what it is given, here without a GPU."""
    import torch
    from paper_2607_10611_gb300 import fp4, layer_norm
    for x in (torch.zeros(3, 4), torch.zeros(3, 4, dtype=torch.float64), torch.zeros(())):
        with pytest.raises(ValueError, match="CUDA"):
            layer_norm(x)
    with pytest.raises(ValueError, match="tensor"):
        layer_norm([1.0])
    with pytest.raises(ValueError, match="CUDA"):
        fp4.NVFP4Matrix(torch.zeros(32, dtype=torch.uint8), torch.zeros(4, dtype=torch.uint8), 1.0, (1, 64))
