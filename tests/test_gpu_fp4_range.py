"""Tokens times an NVFP4 weight where results come near the ends of binary32's range, whatever the weight's scale: a result that
fits is there, one that does not is infinite."""
import math

import pytest
import torch

from test_gpu_fp4 import BF16, F32, _check, _values, _weight, _x

pytestmark = pytest.mark.gpu

from paper_2607_10611_gb300 import fp4  # noqa: E402

SCALES = [2.0 ** -140, 2.0 ** -100, 1.7 * 2.0 ** -45, 1.3 * 2.0 ** -30, 1.9 * 2.0 ** -10, 2.0 ** -8, 0.75, 1.0, 3.0, 2.0 ** 60, 3.0e38]
SHAPES = [(50, 1056), (50, 1001)]  # on the tensor cores, and one by one
TOKENS = [1, 8, 17, 40]


def _sized(x, w, most):
    """x times the power of two with which the absolute values that any result sums up come up to between most / 2 and most, or x
    to where it is still finite."""
    size = float((x.double().abs() @ _values(w).abs().t()).max())
    e = min(math.floor(math.log2(most / size)), 126 - math.frexp(float(x.abs().max()))[1])
    return (x.double() * 2.0 ** e).to(x.dtype)  # (exact)


@pytest.mark.parametrize("scale", SCALES)
@pytest.mark.parametrize("n,k", SHAPES)
@pytest.mark.parametrize("tokens", TOKENS)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_results_at_the_upper_end(dtype, tokens, n, k, scale):
    w = _weight(n, k, seed=k, scale=scale)
    x = _sized(_x(tokens, k, dtype), w, 3.3e38)
    y = fp4.linear(x, w)
    assert bool(y.isfinite().all())
    _check(y, x, w)


@pytest.mark.parametrize("scale", [s for s in SCALES if s >= 0.75])  # (with smaller ones, x is out of range first)
@pytest.mark.parametrize("n,k", SHAPES)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_results_past_the_upper_end_are_infinite(dtype, n, k, scale):
    """All weights and tokens of one sign, so that no partial sum is larger than its result: 8 times the largest number."""
    w = _weight(n, k, seed=k, scale=scale)
    w.codes.bitwise_and_(0x77).bitwise_or_(0x11)  # at least 0.5
    for tokens in TOKENS:
        x = _x(tokens, k, dtype).abs() + 0.5
        least = float((x.double() @ _values(w).t()).min())
        e = math.ceil(math.log2(8 * 3.4e38 / least))
        x = (x.double() * 2.0 ** e).to(dtype)
        assert bool(x.isfinite().all())
        assert bool((fp4.linear(x, w) == math.inf).all())


@pytest.mark.parametrize("scale", SCALES[1:8])
@pytest.mark.parametrize("n,k", SHAPES)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_results_near_the_lower_end(dtype, n, k, scale):
    """Of about 2^-90, so that addends a million times smaller are whole numbers of 2^-149 still."""
    w = _weight(n, k, seed=k, scale=scale)
    for tokens in TOKENS:
        x = _sized(_x(tokens, k, dtype), w, 2.0 ** -90)
        _check(fp4.linear(x, w), x, w)
