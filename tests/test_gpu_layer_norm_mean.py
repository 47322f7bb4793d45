"""The layer norm's statistics where the mean is far from 0: the mean is off by its own last rounding and what the deviations'
sum rounds, whatever its size, and y and the gradients by what that makes of them."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2607_10611_gb300 import layer_norm  # noqa: E402

U = 2.0 ** -24  # a binary32 rounding, relative
BF16, F32 = torch.bfloat16, torch.float32
# a row in a warp's registers, a block's with 8 and more values a thread, with and without packs, wider ones, and rows in turn
SIZES = [(40, 100), (40, 255), (40, 256), (40, 768), (3000, 768), (20000, 768), (900, 1001), (700, 4096), (1300, 4096), (1300, 5632),
         (40, 8191), (40, 8192), (50, 9001), (50, 20000)]


def _inputs(rows, cols, dtype, far):
    g = torch.Generator(device="cuda").manual_seed(rows + cols)
    normal = lambda *s: torch.randn(*s, generator=g, device="cuda")
    x = (normal(rows, cols) + far * (1 + torch.rand(rows, 1, generator=g, device="cuda"))).to(dtype)
    return x, 1 + 0.3 * normal(cols), normal(cols), normal(rows, cols).to(dtype)


def _exact(x):
    """(mean, deviations, K, what binary32 may add to the mean beside its own last rounding, to each deviation, and what the
    first mean may be off by): K roundings bound a sum over a row, as a thread adds at most 32 values, a warp 5 times, a block 16
    (wider rows: cols / 512 in a thread).  The first mean is off by at most (K + 2) U |mean|.  Binary32: what it leaves is added
    up as deviations are, which are rounded once, and summed and divided with K + 2 roundings; it is taken off with one.
    BF16: rows far from 0 here are whole multiples of their smallest value's last place, and their sum one below 2^24 of it (of
    20000 at 60000, 2^7 each, 9.4e6), so exact; what the division leaves is then known but for three roundings.  Rows around 0 are
    not, and keep the sum's error."""
    K = 60 + x.shape[1] // 512
    v = x.double()
    mean = v.mean(1, keepdim=True)
    d = v - mean
    left = (K + 2) * U * v.abs().mean(1, keepdim=True)
    off = (K + 3) * U * (d.abs().mean(1, keepdim=True) + 2 * left)
    if x.dtype == BF16:
        off = off + (v.abs().mean(1, keepdim=True) < 100) * left
    return mean, d, K, off, 2 * U * (d.abs() + 2 * left) + off, left


def _off(got, want, bound):
    half_step = torch.finfo(got.dtype).eps / 2
    return float(((got.double() - want).abs() - (bound * (1 + half_step) + want.abs() * half_step)).max())


@pytest.mark.parametrize("far", [0.0, 1.0, 1000.0, 30000.0])
@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_the_statistics(dtype, rows, cols, far):
    from paper_2607_10611_gb300 import _native as N
    x, w, b, _ = _inputs(rows, cols, dtype, far)
    y, mean, rstd = torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    p = N.mpadam_layer_norm(x.data_ptr(), cols, w.data_ptr(), b.data_ptr(), y.data_ptr(), cols, mean.data_ptr(), rstd.data_ptr(), rows,
                            cols, N.MPADAM_F32 if dtype == F32 else N.MPADAM_BF16, N.MPADAM_F32, 1e-5, 0)
    N.mpadam_layer_norm_forward(p, torch.cuda.current_stream().cuda_stream)
    want, d, K, off, d_d, left = _exact(x)
    # (its own last rounding is _off's half step of binary32)
    assert _off(mean, want[:, 0], off[:, 0]) <= 0
    var = d.square().mean(1)
    # squares of the deviations from the first mean, less the square of what that was off by
    d_var = (K + 6) * U * (var + left[:, 0].square()) + 2 * (d.abs() * d_d).mean(1)
    exact = 1 / (var + 1e-5).sqrt()
    assert _off(rstd, exact, exact * (4 * U + d_var / (var + 1e-5))) <= 0


@pytest.mark.parametrize("far", [1000.0, 30000.0])
@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_outputs_and_gradients(dtype, rows, cols, far):
    x, w, b, dy = _inputs(rows, cols, dtype, far)
    leaves = [t.requires_grad_() for t in (x, w, b)]
    y = layer_norm(*leaves)
    dx, dw, db = torch.autograd.grad(y, leaves, dy)
    x, w, b, dy = (t.detach().double() for t in (x, w, b, dy))
    mean, d, K, off, d_d, left = _exact(x)
    var = d.square().mean(1, keepdim=True)
    rstd = 1 / (var + 1e-5).sqrt()
    n = d * rstd
    d_rstd = 4 * U + ((K + 6) * U * (var + left.square()) + 2 * (d.abs() * d_d).mean(1, keepdim=True)) / (var + 1e-5)
    d_n = d_d * rstd + n.abs() * (d_rstd + 2 * U)
    assert _off(y.detach(), n * w + b, w.abs() * d_n + 3 * U * ((n * w).abs() + b.abs())) <= 0
    # the backward pass takes the mean as it is stored, once rounded
    d_n = d_n + (U * mean.abs() + off) * rstd
    dn = dy * w
    m0, m1 = dn.mean(1, keepdim=True), (dn * n).mean(1, keepdim=True)
    d_m1 = K * U * (dn * n).abs().mean(1, keepdim=True) + (dn.abs() * d_n).mean(1, keepdim=True)
    d_dx = rstd * (K * U * dn.abs().mean(1, keepdim=True) + n.abs() * d_m1 + d_n * m1.abs()
                   + 8 * U * (dn.abs() + m0.abs() + (n * m1).abs()))
    want = (dn - m0 - n * m1) * rstd
    assert _off(dx, want, d_dx + want.abs() * (d_rstd + 2 * U)) <= 0
    R = rows + 48
    assert _off(dw, (dy * n).sum(0), R * U * (dy * n).abs().sum(0) + (dy.abs() * d_n).sum(0)) <= 0
    assert _off(db, dy.sum(0), R * U * dy.abs().sum(0)) <= 0


@pytest.mark.parametrize("cols", [100, 256, 768, 1001, 4096, 9001])
@pytest.mark.parametrize("dtype,size,eps", [(F32, 0.1, 1e-12), (F32, 3000.0, 1e-5), (BF16, 0.1, 1e-12), (BF16, 3000.0, 1e-5)])
def test_rows_of_one_value(dtype, size, eps, cols):
    """Deviations are 0, though the first mean is off: y is the bias, to what is left of n.  The first mean is off by at most
    K + 2 < 80 roundings, 5e-6 of the value, and that is taken off to 4 U of itself: 1.2e-12 of the value, beside rstd of at most
    1 / sqrt(eps): 1.2e-7 and 1.2e-6."""
    x = torch.full((33, cols), size, device="cuda") * torch.arange(1, 34, device="cuda")[:, None] / 33
    b = torch.randn(cols, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).to(dtype)
    y = layer_norm(x.to(dtype), torch.ones(cols, dtype=dtype, device="cuda"), b, eps=eps)
    assert float(((y - b).abs() - b.abs() * torch.finfo(dtype).eps).max()) <= 2e-6
