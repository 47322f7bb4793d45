"""The 8-bit linear layer's operators against plain references: codes and scales bit for bit, products exactly where
binary32 holds every partial sum, else within a bound on its roundings, gradients against the formula and differences."""
import numpy as np
import pytest
import torch

import fp8_reference as R

pytestmark = pytest.mark.gpu

from paper_2607_10611_gb300 import fp8  # noqa: E402


@pytest.fixture(autouse=True)
def waits_held():
    yield
    if torch.cuda.is_available():
        assert fp8.device_status() == 0


def _values(rows, cols, seed, kind="normal"):
    g = np.random.default_rng(seed)
    x = g.normal(0, 1, (rows, cols)).astype(np.float32)
    if kind == "spread":  # block maxima over the whole range of binary32, subnormal ones too
        x *= np.exp2(g.uniform(-148, 120, (rows, -(-cols // 64)))).repeat(64, 1)[:, :cols].astype(np.float32)
    elif kind == "special":
        flat = x.reshape(-1)
        pick = g.permutation(flat.size)
        for i, v in enumerate((0.0, -0.0, np.inf, -np.inf, np.nan, 448.0, 3.4e38, 1e-45)):
            flat[pick[i * flat.size // 20:(i + 1) * flat.size // 20]] = v
        x[: rows // 3] = 0.0
    return x


def _check(q, codes, k):
    assert torch.equal(q.codes.view(torch.uint8).cpu(), torch.from_numpy(codes))
    assert torch.equal(q.scales.view(torch.uint8).cpu(), torch.from_numpy(R.stored_scales(k)))


@pytest.mark.parametrize("square", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols,kind", [
    (1, 1, "normal"), (1, 128, "normal"), (1, 4096, "spread"), (128, 1, "normal"), (3, 130, "special"),
    (127, 129, "spread"), (128, 128, "normal"), (129, 127, "special"), (200, 513, "spread"), (257, 640, "normal"),
    (300, 1030, "special")])
def test_quantize(rows, cols, kind, dtype, square):
    x = torch.from_numpy(_values(rows, cols, rows * 31 + cols, kind)).to(dtype)
    host = x.float().numpy()
    q, qt = fp8.quantize(x.cuda(), square=square, transposed=True)
    _check(q, *R.quantize(host, square))
    _check(qt, *R.quantize(np.ascontiguousarray(host.T), square))
    _check(fp8.quantize(x.cuda(), square=square), *R.quantize(host, square))
    only = fp8.quantize(x.cuda(), square=square, transposed="only")
    assert torch.equal(only.codes.view(torch.uint8), qt.codes.view(torch.uint8))
    assert torch.equal(only.scales.view(torch.uint8), qt.scales.view(torch.uint8))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("first,stride", [(0, 333), (1, 334), (3, 400), (8, 336)])
def test_quantize_takes_strided_rows(first, stride, dtype):
    store = torch.from_numpy(_values(150, stride, 5)).to(dtype)
    x = store[:, first:first + 300]
    q, qt = fp8.quantize(store.cuda()[:, first:first + 300], transposed=True)
    _check(q, *R.quantize(x.float().numpy(), False))
    _check(qt, *R.quantize(np.ascontiguousarray(x.float().numpy().T), False))


def test_values_stand_for_the_codes():
    x = torch.from_numpy(_values(140, 300, 3))
    q = fp8.quantize(x.cuda())
    codes, k = R.quantize(x.numpy(), False)
    want = np.ldexp(R.e4m3_value(codes), k.repeat(128, 1)[:, :300])
    assert np.array_equal(q.dequantize().cpu().double().numpy(), want)
    assert float((q.dequantize().cpu() - x).norm() / x.norm()) < 2 ** -4  # half of E4M3's largest spacing


def _exact_operands(m, n, k, seed):
    """Small whole numbers times powers of two per block: every partial sum is exact in binary32.  |values| reach 4,
    which E4M3 holds, scales reach 2^3, and 4 * 4 * 2^6 * k stays below 2^24 for k <= 16384."""
    g = torch.Generator().manual_seed(seed)
    out = []
    for rows in (m, n):
        v = torch.randint(-4, 5, (rows, k), generator=g).float()
        e = torch.randint(0, 4, (rows, -(-k // 128)), generator=g)
        out.append((v, e))
    return out


def _as_matrix(v, e):
    rows, cols = v.shape
    store = torch.full((rows, -(-cols // 16) * 16), float("nan")).to(fp8.E4M3)  # padding is never used
    store[:, :cols] = v.to(fp8.E4M3)
    s = torch.from_numpy(R.stored_scales(e.numpy())).view(fp8.E8M0)
    return fp8.E4M3Matrix(store.cuda()[:, :cols], s.cuda())


def _value(v, e):
    return v.double() * torch.exp2(e.double()).repeat_interleave(128, 1)[:, :v.shape[1]]


SHAPES = [(1, 1, 1), (1, 128, 128), (2, 300, 16), (3, 5, 7), (8, 4096, 640), (16, 129, 513), (17, 130, 600), (32, 64, 2048),
          (33, 257, 129), (64, 100, 1000), (65, 257, 1000), (100, 4096, 384), (128, 128, 4096), (129, 300, 127),
          (200, 1000, 640), (255, 128, 2048), (256, 256, 512), (257, 384, 4097), (300, 129, 16000), (1000, 1001, 1003),
          (2049, 130, 260), (520, 5000, 300)]


# Pairs of CTAs with tiles of 256 and of 192 rows of a: several tiles a pair, tiles that start inside a scale tile, edges.
SHAPES += [(1920, 2560, 512), (1925, 2550, 900), (2816, 2560, 130), (5000, 1100, 1537), (1023, 5632, 300),
           (4864, 4096, 260), (2048, 2050, 700), (4100, 4100, 140)]


@pytest.mark.parametrize("m,n,k", SHAPES)
def test_product_of_whole_numbers_is_exact(m, n, k):
    (va, ea), (vb, eb) = _exact_operands(m, n, k, m + 7 * n + 13 * k)
    a, b = _as_matrix(va, ea), _as_matrix(vb, eb)
    want = _value(va, ea) @ _value(vb, eb).t()
    assert torch.equal(fp8.matmul(a, b, out_dtype=torch.float32).cpu(), want.float())
    assert torch.equal(fp8.matmul(a, b).cpu(), want.float().to(torch.bfloat16))
    store = torch.full((m, n + 5), 8.0, device="cuda")  # a strided output, its padding left alone
    fp8.matmul(a, b, out=store[:, :n], accumulate=True)
    assert torch.equal(store[:, :n].cpu(), (want + 8.0).float())
    assert bool((store[:, n:] == 8.0).all())


@pytest.mark.parametrize("m,n,k", [(1, 1000, 4096), (40, 300, 16384), (300, 300, 8119), (1024, 768, 2304)])
def test_product_of_real_values(m, n, k):
    """Every 32 values of k are added to the sum with at most one rounding or truncation each of the sum and of the
    aligned addends: 2 k / 32 times 2^-23 of the sum of magnitudes bounds the error of a binary32 result."""
    g = torch.Generator().manual_seed(k)
    a = torch.randn(m, k, generator=g) + 0.3
    b = torch.randn(n, k, generator=g) * torch.exp(torch.randn(k, generator=g)) + 0.1
    qa, qb = fp8.quantize(a.cuda()), fp8.quantize(b.cuda())
    va, vb = qa.dequantize().double(), qb.dequantize().double()
    want, size = va @ vb.t(), va.abs() @ vb.abs().t()
    got = fp8.matmul(qa, qb, out_dtype=torch.float32).double()
    assert bool(((got - want).abs() <= (2 * -(-k // 32) + 1) * 2.0 ** -23 * size).all())
    low = fp8.matmul(qa, qb).double()
    assert bool(((low - got).abs() <= 2.0 ** -8 * got.abs()).all())
    assert torch.equal(fp8.matmul(qa, qb, out_dtype=torch.float32).double(), got)  # the same bits every time


def test_scales_over_their_whole_range():
    v = torch.ones(130, 256)
    for ea, eb in ((-127, 120), (120, -127), (-60, -60), (60, 59), (-127, 0)):
        a, b = _as_matrix(v, torch.full((130, 2), ea)), _as_matrix(v, torch.full((130, 2), eb))
        got = fp8.matmul(a, b, out_dtype=torch.float32).cpu()
        assert torch.equal(got, torch.full((130, 130), 256.0 * 2.0 ** (ea + eb)).float())


def test_not_a_number_stays_in_its_row_and_column():
    a, b = torch.ones(150, 300), torch.ones(200, 300)
    a[149, 299] = float("nan")
    b[7, 128] = float("nan")
    got = fp8.matmul(fp8.quantize(a.cuda()), fp8.quantize(b.cuda()), out_dtype=torch.float32).cpu()
    bad = torch.zeros(150, 200, dtype=torch.bool)
    bad[149], bad[:, 7] = True, True
    assert torch.equal(got.isnan(), bad) and bool((got[~bad] == 300.0).all())


def test_empty_sizes():
    for m, n, k in ((0, 4, 16), (4, 0, 16), (3, 5, 0), (0, 0, 0)):
        a, b = fp8.quantize(torch.ones(m, k, device="cuda")), fp8.quantize(torch.ones(n, k, device="cuda"))
        assert torch.equal(fp8.matmul(a, b).cpu(), torch.zeros(m, n, dtype=torch.bfloat16))
        out = torch.ones(m, n, device="cuda")
        assert torch.equal(fp8.matmul(a, b, out=out, accumulate=True).cpu(), torch.ones(m, n))


def _layer(tokens, k, n, seed, dtype=torch.bfloat16):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(tokens, k, generator=g).to(dtype).cuda().requires_grad_()
    w = (0.05 * torch.randn(n, k, generator=g)).to(dtype).cuda().requires_grad_()
    return x, w, torch.randn(tokens, n, generator=g).to(dtype).cuda()


def _quantised(x, square=False):
    """The values of x on its 8-bit grid, in binary64, by the numpy reference."""
    host = x.detach().float().cpu().numpy()
    codes, k = R.quantize(host, square)
    return torch.from_numpy(np.ldexp(R.e4m3_value(codes), k.repeat(128, 1)[:, :host.shape[1]]))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("tokens,k,n", [(1, 64, 96), (37, 200, 130), (256, 512, 384), (515, 130, 1)])
def test_linear_and_its_gradients_by_the_formula(tokens, k, n, dtype):
    x, w, dy = _layer(tokens, k, n, tokens, dtype)
    y = fp8.linear(x, w)
    dx, dw = torch.autograd.grad(y, (x, w), dy)
    qx, qw, qdy = _quantised(x), _quantised(w, True), _quantised(dy)
    qxt, qdyt = _quantised(x.detach().t()), _quantised(dy.t())
    for got, p, q in ((y, qx, qw.t()), (dx, qdy, qw), (dw, qdyt, qxt.t())):
        want, size = p @ q, p.abs() @ q.abs()
        bound = (2 * -(-p.shape[1] // 32) + 1) * 2.0 ** -23 * size
        if dtype == torch.bfloat16:
            bound += 2.0 ** -8 * want.abs()
        assert got.dtype == dtype and got.shape == want.shape
        assert bool(((got.detach().cpu().double() - want).abs() <= bound).all())


def test_gradients_by_differences():
    """Whole numbers that E4M3 holds exactly, in blocks whose scale stays the same: y is then the bilinear x w^T without
    any rounding, and differences give its gradient exactly."""
    g = torch.Generator().manual_seed(0)
    x = torch.randint(-3, 4, (40, 130), generator=g).float()
    w = torch.randint(-3, 4, (30, 130), generator=g).float()
    dy = torch.randint(-3, 4, (40, 30), generator=g).float()
    x[:, 0] = x[:, 128] = w[:, 0] = w[:, 128] = 8.0  # the blocks' maxima
    xg, wg = x.cuda().requires_grad_(), w.cuda().requires_grad_()
    dx, dw = torch.autograd.grad(fp8.linear(xg, wg), (xg, wg), dy.cuda())

    def loss(x, w):
        return float((fp8.linear(x.cuda(), w.cuda()).cpu().double() * dy).sum())

    base = loss(x, w)
    for i, j in ((0, 1), (39, 129), (17, 64), (5, 127)):
        for v, d in ((x, dx), (w, dw)):
            if i < v.shape[0]:
                moved = v.clone()
                moved[i, j] += 1.0
                assert (loss(moved, w) if v is x else loss(x, moved)) - base == float(d[i, j])


def test_linear_leading_dimensions_expanded_gradients_and_partial_needs():
    x, w, _ = _layer(24, 96, 40, 1)
    y = fp8.linear(x.view(2, 3, 4, 96), w)
    assert y.shape == (2, 3, 4, 40)
    dx, dw = torch.autograd.grad(y.sum(), (x, w))  # a gradient whose strides are all zero
    assert torch.equal(dx, torch.autograd.grad(fp8.linear(x, w), x, torch.ones(24, 40, device="cuda", dtype=x.dtype))[0])
    assert torch.equal(dw, torch.autograd.grad(fp8.linear(x.detach(), w).sum(), w)[0])
    assert torch.equal(dx, torch.autograd.grad(fp8.linear(x, w.detach()).sum(), x)[0])
    xt = x.detach().t().contiguous().t()  # columns first
    assert torch.equal(fp8.linear(xt, w.detach()), fp8.linear(x.detach(), w.detach()))


def test_linear_adds_to_the_weight_gradient_it_is_given():
    x, w, dy = _layer(130, 96, 40, 2)
    total = torch.full((40, 96), 0.5, device="cuda")
    for _ in range(2):
        fp8.linear(x, w, grad_w=total).backward(dy)
    want = _quantised(dy.t()) @ _quantised(x.detach().t()).t()
    assert w.grad is None
    assert bool(((total.cpu().double() - 0.5 - 2 * want).abs() <= 1e-5 * (1 + want.abs().max())).all())


def test_graphs_of_the_layer():
    """A second backward pass needs the graph to be retained; a second derivative is refused; an unused output's gradient
    is none; what autograd sees is one node whose inputs are x and w."""
    x, w, dy = _layer(8, 96, 40, 1)
    y = fp8.linear(x, w)
    first = torch.autograd.grad(y, (x, w), dy, retain_graph=True)
    second = torch.autograd.grad(y, (x, w), dy)
    assert all(torch.equal(a, b) for a, b in zip(first, second))
    with pytest.raises(RuntimeError, match="second time"):
        torch.autograd.grad(y, (x, w), dy)
    with pytest.raises(RuntimeError, match="differentiable once"):
        torch.autograd.grad(fp8.linear(x, w).float().square().sum(), x, create_graph=True)
    assert y.grad_fn.name() == "E4M3LinearBackward" and len(y.grad_fn.next_functions) == 2
    h = fp8.linear(x, w)
    z = fp8.linear(torch.nn.functional.gelu(h), w.detach().t().contiguous())  # through another layer
    z.sum().backward()
    assert x.grad is not None and w.grad is not None and z.requires_grad and not fp8.linear(x.detach(), w.detach()).requires_grad


@pytest.mark.parametrize("xt,wt", [(torch.float32, torch.bfloat16), (torch.bfloat16, torch.float32)])
def test_activations_and_weights_of_different_types(xt, wt):
    """The result and dx have x's type, dw has w's; each rounds once from the same binary32 product."""
    x, w, dy = _layer(40, 160, 56, 4, torch.float32)
    x, w = x.detach().to(xt).requires_grad_(), w.detach().to(wt).requires_grad_()
    dy = dy.to(xt)
    y = fp8.linear(x, w)
    dx, dw = torch.autograd.grad(y, (x, w), dy)
    assert (y.dtype, dx.dtype, dw.dtype) == (xt, xt, wt)
    x32, w32 = x.detach().float().requires_grad_(), w.detach().float().requires_grad_()
    y32 = fp8.linear(x32, w32)
    dx32, dw32 = torch.autograd.grad(y32, (x32, w32), dy.float())
    assert torch.equal(y, y32.to(xt)) and torch.equal(dx, dx32.to(xt)) and torch.equal(dw, dw32.to(wt))


def test_inference_mode_gives_the_same():
    x, w, _ = _layer(24, 160, 56, 4)
    want = fp8.linear(x, w).detach()
    with torch.inference_mode():
        held = fp8.quantize(w, square=True)
        assert torch.equal(fp8.linear(x, w), want) and torch.equal(fp8.linear(x, held), want)
        assert torch.equal(fp8.linear(x.clone(), w.clone()), want)


def test_linear_of_no_tokens():
    x, w, dy = _layer(0, 96, 40, 1)
    for shape in ((0, 96), (2, 0, 96)):
        y = fp8.linear(x.view(shape), w)
        assert y.shape == (*shape[:-1], 40)
        dx, dw = torch.autograd.grad(y, (x, w), torch.zeros_like(y))
        assert dx.shape == (0, 96) and torch.equal(dw, torch.zeros_like(dw))


@pytest.mark.parametrize("tokens", [1, 5, 40])
def test_serving_with_a_held_weight_gives_the_same(tokens):
    x, w, _ = _layer(tokens, 512, 700, 3)
    with torch.no_grad():
        held = fp8.quantize(w, square=True)
        assert torch.equal(fp8.linear(x, held), fp8.linear(x, w))


@pytest.mark.parametrize("tokens,k,n", [(1, 4096, 1024), (20, 512, 3000), (100, 2048, 500)])
def test_a_weight_written_just_before_it_serves(tokens, k, n):
    """The weight's copies begin while the tokens are quantised, not before what wrote the weight has ended; and what
    follows on the stream sees the product."""
    x, w, _ = _layer(tokens, k, n, 6)
    x, w = x.detach(), w.detach()
    got, want = [], []
    for i in range(30):
        w = w.roll(1, 0)
        held = fp8.quantize(w, square=True)
        got.append(fp8.linear(x, held))
        got[-1] += 1.0
    torch.cuda.synchronize()
    for i in range(30):
        w = w.roll(-1, 0) if i else w
        want.insert(0, fp8.linear(x, w) + 1.0)
        torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_other_streams_and_graphs():
    x, w, _ = _layer(70, 256, 200, 4)
    x, w = x.detach(), w.detach()
    want = fp8.linear(x, w)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = fp8.linear(x, w)
    q = fp8.quantize(x, stream=side)
    qw = fp8.quantize(w, square=True, stream=side)
    again = fp8.matmul(q, qw, stream=side)
    side.synchronize()
    assert torch.equal(got, want) and torch.equal(again, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = fp8.linear(x, w)
    x.neg_()
    graph.replay()
    assert torch.equal(out, -want)


def test_refusals():
    x = torch.ones(4, 32, device="cuda")
    q = fp8.quantize(x)
    with pytest.raises(ValueError):
        fp8.quantize(x.half())
    with pytest.raises(ValueError):
        fp8.quantize(x.t())  # its rows are not contiguous
    with pytest.raises(ValueError):
        fp8.quantize(x[0].expand(4, 32))  # rows that share memory
    with pytest.raises(ValueError):
        fp8.quantize(x, transposed="yes")
    with pytest.raises(ValueError):
        fp8.matmul(q, fp8.quantize(x[:, :16].contiguous()))
    with pytest.raises(ValueError):
        fp8.matmul(q, q, accumulate=True)
    with pytest.raises(ValueError):
        fp8.matmul(q, q, out=torch.empty(4, 5, device="cuda"))
    with pytest.raises(ValueError):
        fp8.E4M3Matrix(q.codes, q.scales[:, :, :16])
    with pytest.raises(ValueError):
        fp8.linear(x.requires_grad_(), q)
    codes = torch.zeros(4, 40, dtype=torch.uint8, device="cuda").view(fp8.E4M3)[:, :32]
    with pytest.raises(RuntimeError, match="multiples of 16"):  # rows 40 bytes apart
        fp8.matmul(fp8.E4M3Matrix(codes, q.scales), q)
    with pytest.raises(RuntimeError, match="binary32"):
        fp8.matmul(q, q, out=torch.zeros(4, 4, dtype=torch.bfloat16, device="cuda"), accumulate=True)
