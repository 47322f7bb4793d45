"""Refusals of the AdamW, gradient-norm and 8-bit matrix entry points that are decided on the host, before any CUDA call
(no GPU needed)."""
import math
import random

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


def _config(N, **kw):
    d = dict(beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, weight_dtype=N.MPADAM_BF16, grad_dtype=N.MPADAM_F32,
             state_dtype=N.MPADAM_E4M3, rounding=0, state_rounding=0, reserved=0, seed=0)
    return N.mpadam_adamw_config(**{**d, **kw})


GOOD = (0x1000, 0x2000, 0x3000, 0x4000, 0x5000, 0, 256)


@pytest.mark.parametrize("bad", [
    dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=math.nan), dict(eps=0.0), dict(eps=math.inf), dict(weight_decay=-1.0),
    dict(weight_dtype=2), dict(grad_dtype=2), dict(state_dtype=1), dict(rounding=2), dict(state_rounding=-1),
    dict(reserved=1), dict(state_dtype=0, state_rounding=1)])
def test_adamw_refuses_bad_configs(N, bad):
    refused(N, N.mpadam_adamw_create, [GOOD], _config(N, **bad))


@pytest.mark.parametrize("at,value", [(0, 0), (1, 0), (2, 0), (3, 0), (4, 0), (0, 0x1001), (5, 0x7000), (6, -1)])
def test_adamw_refuses_bad_tensors(N, at, value):
    t = list(GOOD)
    t[at] = value  # (a BF16 weight has no compute copy)
    refused(N, N.mpadam_adamw_create, [GOOD, tuple(t)], _config(N))


def test_adamw_refuses_misaligned_binary32_moments_and_their_scales(N):
    refused(N, N.mpadam_adamw_create, [(0x1000, 0x2002, 0x3000, 0, 0, 0, 8)], _config(N, state_dtype=N.MPADAM_F32))
    refused(N, N.mpadam_adamw_create, [GOOD], _config(N, state_dtype=N.MPADAM_F32))


def test_norm_refuses(N):
    refused(N, N.mpadam_grad_norm_create, [-1], N.MPADAM_F32)
    refused(N, N.mpadam_grad_norm_create, [1], N.MPADAM_E4M3)


def test_null_handles_are_refused_and_their_destruction_is_not(N):
    refused(N, N.mpadam_adamw_step, 0, [0x1000], 1, 1e-3)
    refused(N, N.mpadam_grad_norm, 0, [0x1000], 1.0, 0x1000)
    N.mpadam_adamw_destroy(0)
    N.mpadam_grad_norm_destroy(0)


QUANT = dict(x=0x1000, x_dtype=0, rows=4, cols=20, ld=20, square=0, q=0x2000, s=0x3000, ldq=32, qt=0x4000, st=0x5000, ldqt=16)


@pytest.mark.parametrize("bad", [
    dict(x_dtype=2), dict(rows=-1), dict(cols=1 << 31), dict(ld=19), dict(square=2), dict(x=0), dict(x=0x1002),
    dict(q=0x2008), dict(s=0), dict(s=0x3004), dict(ldq=16), dict(ldq=24), dict(qt=0x4001), dict(st=0), dict(ldqt=2),
    dict(ldqt=0), dict(q=0, qt=0), dict(rows=(1 << 31) - 1, cols=(1 << 31) - 1, ld=1 << 31, ldq=1 << 31, ldqt=1 << 31)])
def test_quantize_refuses(N, bad):
    refused(N, N.mpadam_e4m3_quantize, **{**QUANT, **bad})


PRODUCT = dict(a=0x1000, a_scale=0x2000, lda=48, b=0x3000, b_scale=0x4000, ldb=48, d=0x5000, ldd=9, m=5, n=9, k=40,
               d_dtype=0, accumulate=0)


@pytest.mark.parametrize("bad", [
    dict(m=-1), dict(n=1 << 31), dict(k=-1), dict(n=(1 << 31) - 1023, ldd=1 << 31), dict(d_dtype=2), dict(accumulate=2), dict(accumulate=1, d_dtype=1),
    dict(d=None), dict(d=0x5002), dict(ldd=8), dict(a=None), dict(a=0x1008), dict(b_scale=None), dict(a_scale=0x2001),
    dict(lda=32), dict(ldb=40)])
def test_matmul_refuses(N, bad):
    refused(N, N.mpadam_e4m3_matmul, N.mpadam_e4m3_product(**{**PRODUCT, **bad}))


@pytest.mark.parametrize("bad", [dict(ldx=39), dict(x_dtype=2), dict(x=0), dict(a=None), dict(a_scale=None), dict(lda=47),
                                 dict(b=None), dict(b=0x3008), dict(ldb=40), dict(d=None), dict(ldd=8), dict(d_dtype=3),
                                 dict(accumulate=1, d_dtype=1), dict(m=-1)])
def test_quantize_matmul_refuses(N, bad):
    """All before its first launch, the product's arguments too."""
    call = dict(x=0x9000, x_dtype=0, ldx=40)
    call.update({k: v for k, v in bad.items() if k in call})
    product = N.mpadam_e4m3_product(**{**PRODUCT, **{k: v for k, v in bad.items() if k not in call}})
    refused(N, N.mpadam_e4m3_quantize_matmul, **call, product=product)


def test_sizes_of_zero_need_no_pointers(N):
    N.mpadam_e4m3_quantize(**{**QUANT, "rows": 0, "x": 0, "q": 0, "qt": 0})
    N.mpadam_e4m3_matmul(N.mpadam_e4m3_product(**{**PRODUCT, "m": 0, "a": None, "d": None}))


def test_products_are_cut_up_so_that_scales_start_where_they_can(N):
    """Tiles of fewer than 128 rows only for an a that has no more (their scales then start with their scale tile), pairs'
    tiles at multiples of 64 rows; a tile's k shared out only among as many CTAs as there are groups of 512."""
    g = random.Random(0)
    seen = set()
    for _ in range(3000):
        m, n, k = (int(math.exp(g.uniform(0, math.log(20000)))) for _ in range(3))
        tile, split, pair = N.mpadam_debug_e4m3_plan(m, n, k)
        seen.add((tile, pair))
        if pair:
            assert tile in (192, 256) and split == 1
        else:
            assert tile == 128 or m <= tile
            assert split in (1, 2, 4, 8) and split <= max(1, -(-k // 512))
    assert seen == {(16, False), (32, False), (64, False), (128, False), (192, True), (256, True)}
