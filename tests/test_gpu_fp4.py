"""Tokens times a weight in NVFP4 against the product in 64 bits of what codes and scales stand for: every number of tokens
to a block's tile and beyond, odd sizes and alignments, both types, every code and scale, values that are not finite; and the
weights that M+Adam's step leaves."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2607_10611_gb300 import fp4  # noqa: E402

BF16, F32 = torch.bfloat16, torch.float32


def _weight(n, k, seed=0, scale=2.0 ** -9):
    g = torch.Generator(device="cuda").manual_seed(seed)
    codes = torch.randint(0, 256, ((n * k + 1) // 2,), generator=g, device="cuda", dtype=torch.uint8)
    scales = torch.randint(0x28, 0x58, ((n * k + 15) // 16,), generator=g, device="cuda", dtype=torch.uint8)
    return fp4.NVFP4Matrix(codes, scales, scale, (n, k))


def _values(w):
    """In 64 bits, by each element's own nibble and group."""
    n, k = w.shape
    at = torch.arange(n * k, device="cuda")
    code = (w.codes.reshape(-1)[at // 2].long() >> 4 * (at % 2)) & 15
    e, f = code // 2 % 4, code % 2
    value = torch.where(e > 0, torch.exp2(e.double() - 1) * (1 + f / 2.0), f / 2.0) * (1 - 2 * (code // 8)).double()
    return (value * w.scales.reshape(-1).view(torch.float8_e4m3fn).double()[at // 16] * w.global_scale).view(n, k)


def _x(tokens, k, dtype, seed=1):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(tokens, k, generator=g, device="cuda") * torch.exp(torch.randn(k, generator=g, device="cuda"))).to(dtype)


def _check(y, x, w):
    """Products are exact; a sum in binary32 rounds or truncates at most once for each of its k addends and 8 shares."""
    v = _values(w)
    want, size = x.double() @ v.t(), x.double().abs() @ v.abs().t()
    half_step = torch.finfo(y.dtype).eps / 2
    bound = (x.shape[1] + 16) * 2.0 ** -23 * size
    far = (y.double() - want).abs() - (bound + (want.abs() + bound) * half_step)
    assert y.dtype == x.dtype and y.shape == want.shape and float(far.max()) <= 0
    # and within what such errors come to as a rule
    assert float((y.double() - want).norm()) <= (2e-6 + half_step) * float(size.norm())


@pytest.mark.parametrize("tokens", [1, 2, 3, 4, 7, 8, 9, 15, 16, 17, 24, 31, 32, 33, 70])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_every_number_of_tokens(dtype, tokens):
    w = _weight(200, 1056)
    x = _x(tokens, 1056, dtype)
    y = fp4.linear(x, w)
    _check(y, x, w)
    assert torch.equal(y, fp4.linear(x, w))


@pytest.mark.parametrize("n,k", [(1, 32), (1, 16), (5, 48), (16, 32), (17, 64), (63, 96), (64, 128), (65, 160), (100, 512), (31, 1024),
                                 (33, 2048), (9, 2080), (48, 4096), (40, 11008), (3, 1), (7, 3), (5, 15), (9, 17), (11, 100),
                                 (64, 1000), (13, 4099)])
@pytest.mark.parametrize("tokens", [1, 5, 20])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_sizes(dtype, tokens, n, k):
    w = _weight(n, k, seed=n + k)
    x = _x(tokens, k, dtype)
    _check(fp4.linear(x, w), x, w)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_every_code_and_scale(dtype):
    """All 16 codes times all 127 finite scales and their negatives, one at a time: exact results."""
    scales = torch.tensor([c for c in range(256) if c & 127 != 127], dtype=torch.uint8, device="cuda")
    n = scales.numel()
    half = torch.arange(16, device="cuda") * 1
    nibbles = half.repeat(2 * n).to(torch.uint8).view(-1, 2)
    w = fp4.NVFP4Matrix((nibbles[:, 0] | nibbles[:, 1] << 4).contiguous(), scales.repeat_interleave(2), 0.75, (n, 32))
    for cols in (32, 31):
        if cols == 31:  # the other kernel, from a flat weight of rows of 31
            flat = torch.nn.functional.pad(_nibbles(w)[:, :31].reshape(-1), (0, n * 31 % 2))
            codes = (flat[0::2] | flat[1::2] << 4).contiguous()
            w = fp4.NVFP4Matrix(codes, scales.repeat_interleave(2)[:(n * 31 + 15) // 16].contiguous(), 0.75, (n, 31))
        eye = torch.eye(cols, device="cuda").to(dtype)
        want = _values(w).t().to(dtype)  # (q s G has 2 + 4 + 2 bits: both types hold it)
        assert torch.equal(fp4.linear(eye, w), want)
        assert torch.equal(w.dequantize().t().to(dtype), want)


def _nibbles(w):
    return torch.stack([w.codes & 15, w.codes >> 4], 1).view(w.shape)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_strides_and_alignment(dtype):
    n, k = 50, 320
    w, x = _weight(n, k), _x(6, k, dtype)
    want = fp4.linear(x, w)
    padded = torch.empty(6, k + 40, dtype=dtype, device="cuda")[:, 8:8 + k].copy_(x)
    off = torch.empty(6 * k + 1, dtype=dtype, device="cuda")[1:].view(6, k).copy_(x)
    for other in (padded, off, x.t().contiguous().t(), x.view(2, 3, k)):
        assert torch.equal(fp4.linear(other, w).view(6, n), want)
    assert torch.equal(fp4.linear(x[2], w), fp4.linear(x[2:3], w)[0])
    # codes and scales off their boundaries take the other kernel
    codes = torch.empty(w.codes.numel() + 3, dtype=torch.uint8, device="cuda")[3:].copy_(w.codes)
    scales = torch.empty(w.scales.numel() + 1, dtype=torch.uint8, device="cuda")[1:].copy_(w.scales)
    for moved in (fp4.NVFP4Matrix(codes, w.scales, w.global_scale, (n, k)), fp4.NVFP4Matrix(w.codes, scales, w.global_scale, (n, k))):
        _check(fp4.linear(x, moved), x, moved)
    assert torch.equal(fp4.linear(x, fp4.NVFP4Matrix(w.codes.view(n, k // 2), w.scales.view(torch.float8_e4m3fn).view(n, k // 16),
                                                     w.global_scale, (n, k))), want)


@pytest.mark.parametrize("k", [64, 63])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_values_that_are_not_finite(dtype, k):
    """They reach their own token, and every row that multiplies them."""
    w, x = _weight(20, k), _x(5, k, dtype)
    w.codes.fill_(0x22)  # ones
    clean = fp4.linear(x, w)
    x[1, 3], x[3, 7], x[4, 0] = float("nan"), float("inf"), float("-inf")
    y = fp4.linear(x, w)
    assert torch.equal(y[[0, 2]], clean[[0, 2]])
    assert bool(y[1].isnan().all()) and bool((y[3] == float("inf")).all()) and bool((y[4] == float("-inf")).all())
    w.scales[0] = 0x7F
    y = fp4.linear(x, w)
    assert bool(y[:, 0].isnan().all()) and torch.equal(y[:, 1:][[0, 2]][:, 1:], clean[[0, 2]][:, 2:])


def test_binary32_keeps_its_bits():
    """Its 24 bits go through the tensor cores in three parts: single products are exact."""
    w = _weight(8, 32)
    w.codes.fill_(0)
    w.codes.view(8, 16)[:, 4] = 2  # element 8 of each row is 1
    w.scales.fill_(0x38)
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.zeros(200, 32, device="cuda")
    x[:, 8] = torch.randn(200, generator=g, device="cuda") * torch.exp2(torch.randint(-60, 60, (200,), generator=g, device="cuda").float())
    assert torch.equal(fp4.linear(x, w), (x[:, 8] * w.global_scale)[:, None].expand(200, 8))


def test_what_the_step_trained():
    """M+Adam's own compute copy of NVFP4 weights and the product with the weights themselves."""
    from paper_2607_10611_gb300 import MPAdam
    n, k = 96, 160
    g = torch.Generator(device="cuda").manual_seed(0)
    codes = torch.randint(0, 256, (n * k // 2,), generator=g, device="cuda", dtype=torch.uint8)
    scales = torch.full((n * k // 16,), 0x38, dtype=torch.uint8, device="cuda")
    moments = [torch.zeros(n * k, device="cuda") for _ in range(3)]
    copy = torch.empty(n, k, dtype=BF16, device="cuda")
    opt = MPAdam([codes], *([m] for m in moments), weight_dtype=["nvfp4"], block_scales=[scales], compute=[copy],
                 global_scales=[2.0 ** -8], grad_dtype="f32")
    w = fp4.NVFP4Matrix(codes, scales, 2.0 ** -8, (n, k))
    before = fp4.linear(torch.eye(k, device="cuda").to(BF16), w)
    for t in (1, 2):
        opt.step([torch.randn(n * k, generator=g, device="cuda")], t)
        y = fp4.linear(torch.eye(k, device="cuda").to(BF16), w)
        assert torch.equal(y.t(), copy)
    assert not torch.equal(y, before)


def test_captured_on_another_stream_and_replayed():
    w, x = _weight(300, 512), _x(4, 512, BF16)
    want = fp4.linear(x, w)
    static = torch.zeros_like(x)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = fp4.linear(static, w)
    static.copy_(x)
    graph.replay()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = fp4.linear(x, w)
    torch.cuda.synchronize()
    assert torch.equal(y, want) and torch.equal(other, want)


def test_nothing_and_refusals():
    w, x = _weight(6, 64), _x(3, 64, BF16)
    assert fp4.linear(x[:0], w).shape == (0, 6)
    empty = torch.empty(0, dtype=torch.uint8, device="cuda")
    assert fp4.linear(x, fp4.NVFP4Matrix(empty, empty, 1.0, (0, 64))).shape == (3, 0)
    y = fp4.linear(x[:, :0], fp4.NVFP4Matrix(empty, empty, 1.0, (6, 0)))
    assert y.shape == (3, 6) and not y.any()
    for make in (lambda: fp4.NVFP4Matrix(w.codes[:-1], w.scales, 1.0, (6, 64)), lambda: fp4.NVFP4Matrix(w.codes, w.scales[:-1], 1.0, (6, 64)),
                 lambda: fp4.NVFP4Matrix(w.codes, w.scales.cpu(), 1.0, (6, 64)), lambda: fp4.NVFP4Matrix(w.codes, w.scales, 0.0, (6, 64)),
                 lambda: fp4.NVFP4Matrix(w.codes, w.scales, float("nan"), (6, 64)),
                 lambda: fp4.NVFP4Matrix(w.codes, w.scales, float("inf"), (6, 64)),
                 lambda: fp4.NVFP4Matrix(w.codes, w.scales.float(), 1.0, (6, 64)),
                 lambda: fp4.NVFP4Matrix(w.codes, w.scales, 1.0, (-6, -64)),
                 lambda: fp4.linear(x[:, :32], w), lambda: fp4.linear(x.half(), w), lambda: fp4.linear(x.cpu(), w),
                 lambda: fp4.linear(x.clone().requires_grad_(), w)):
        with pytest.raises(ValueError):
            make()
    with torch.no_grad():
        fp4.linear(x.clone().requires_grad_(), w)
    with torch.autograd.forward_ad.dual_level():
        with pytest.raises(RuntimeError, match="forward-mode"):
            fp4.linear(torch.autograd.forward_ad.make_dual(x, torch.ones_like(x)), w)


@pytest.mark.parametrize("n,k", [(16, 11008), (40, 4096), (576, 11008), (1000, 2112), (64, 32768), (4096, 640), (33, 1024)])
@pytest.mark.parametrize("tokens", [1, 6, 9, 17, 25, 40])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_too_few_for_all_sms(dtype, tokens, n, k):
    """k is shared out inside a cluster of two, four or eight blocks."""
    w, x = _weight(n, k), _x(tokens, k, dtype)
    y = fp4.linear(x, w)
    _check(y, x, w)
    assert torch.equal(y, fp4.linear(x, w))


@pytest.mark.parametrize("tokens", [1, 3, 8, 11, 24])
def test_what_lies_behind_the_last_token_and_row_stays(tokens):
    from paper_2607_10611_gb300 import _native as N
    n, k, ld = 200, 2080, 208
    w, x = _weight(n, k), _x(tokens, k, BF16)
    y = torch.full((tokens + 2, ld), 8.0, dtype=BF16, device="cuda")
    m = N.mpadam_nvfp4_matrix(w.codes.data_ptr(), w.scales.data_ptr(), n, k, w.global_scale, 0)
    N.mpadam_nvfp4_linear(x.data_ptr(), N.MPADAM_BF16, tokens, k, m, y.data_ptr(), ld, torch.cuda.current_stream().cuda_stream)
    assert torch.equal(y[:tokens, :n], fp4.linear(x, w))
    assert bool((y[tokens:] == 8.0).all()) and bool((y[:, n:] == 8.0).all())


@pytest.mark.parametrize("tokens", [2, 12])
def test_offsets_past_32_bits(tokens):
    n, k = 1050000, 4128
    assert n * k > 2 ** 32
    w, x = _weight(n, k), _x(tokens, k, BF16)
    y = fp4.linear(x, w)
    last = 40  # rows, as a matrix of their own: whole bytes and groups, since k is a multiple of 32
    tail = fp4.NVFP4Matrix(w.codes[-last * k // 2:].clone(), w.scales[-last * k // 16:].clone(), w.global_scale, (last, k))
    _check(y[:, -last:].contiguous(), x, tail)
