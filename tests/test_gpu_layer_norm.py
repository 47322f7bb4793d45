"""Layer normalisation, forward and backward, against its formulas in 64 bits: every path by width (a warp's rows, a block's,
wider ones), odd widths, strides and alignment, types, values far from 0, rows that are not finite; and its place in torch's
graph."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2607_10611_gb300 import layer_norm  # noqa: E402

U = 2.0 ** -24  # a binary32 rounding, relative
BF16, F32 = torch.bfloat16, torch.float32


def _inputs(rows, cols, dtype, wdtype, seed=0, mean=0.5):
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *s: torch.randn(*s, generator=g, device="cuda")
    x = ((normal(rows, cols) + mean) * torch.exp(normal(rows, 1))).to(dtype)
    w, b = (1 + 0.3 * normal(cols)).to(wdtype), normal(cols).to(wdtype)
    return x, w, b, normal(rows, cols).to(dtype)


def _reference(x, w, b, dy, eps):
    """(y, dx, dw, db) in 64 bits and bounds of what binary32 arithmetic may add to each.  A sum over a row is at most 32
    additions in a thread, 5 in a warp and 16 over warps (wider rows: cols / 512 in a thread), so K roundings bound it."""
    rows, cols = x.shape
    K = 60 + cols // 512
    x, w, b, dy = (t.double() for t in (x, w, b, dy))
    mean = x.mean(1, keepdim=True)
    var = (x - mean).square().mean(1, keepdim=True)
    rstd = 1 / (var + eps).sqrt()
    n = (x - mean) * rstd
    # n: the mean's error and the difference's, then rstd's (half of the variance's, and the root's and quotient's)
    d_mean = K * U * x.abs().mean(1, keepdim=True)
    d_n = (d_mean + U * (x.abs() + mean.abs())) * rstd * 2 + n.abs() * (K + 8) * U
    y = n * w + b
    d_y = w.abs() * d_n + 3 * U * ((n * w).abs() + b.abs())
    dn = dy * w
    a0, a1 = dn.abs().mean(1, keepdim=True), (dn * n).abs().mean(1, keepdim=True)
    m0, m1 = dn.mean(1, keepdim=True), (dn * n).mean(1, keepdim=True)
    dx = (dn - m0 - n * m1) * rstd
    d_m1 = K * U * a1 + (dn.abs() * d_n).mean(1, keepdim=True)
    d_dx = rstd * (K * U * a0 + n.abs() * d_m1 + d_n * m1.abs() + 8 * U * (dn.abs() + m0.abs() + (n * m1).abs())) \
        + dx.abs() * (K + 8) * U
    # over rows: each of them at most one addition after another, 8 warps, 32 groups of parts
    R = rows + 48
    dw, db = (dy * n).sum(0), dy.sum(0)
    d_dw = R * U * (dy * n).abs().sum(0) + (dy.abs() * d_n).sum(0)
    d_db = R * U * dy.abs().sum(0)
    return (y, dx, dw, db), (d_y, d_dx, d_dw, d_db)


def _check(got, want, bound, what):
    assert got.shape == want.shape, what
    half_step = torch.finfo(got.dtype).eps / 2
    far = (got.double() - want).abs() - (bound * (1 + half_step) + want.abs() * half_step + 1e-40)
    assert float(far.max()) <= 0 if far.numel() else True, f"{what}: {float(far.max())} past its bound"


def _run(x, w, b, dy, eps):
    leaves = [t.detach().requires_grad_() for t in (x, w, b)]
    y = layer_norm(*leaves, eps=eps)
    return (y.detach(), *torch.autograd.grad(y, leaves, dy))


TYPES = [(BF16, BF16), (BF16, F32), (F32, F32)]
WIDTHS = [1, 2, 7, 8, 31, 64, 100, 255, 256, 264, 512, 513, 768, 1000, 1001, 1024, 1025, 1032, 2048, 4096, 5632, 8191, 8192, 8193,
          8200, 20000]


@pytest.mark.parametrize("cols", WIDTHS)
@pytest.mark.parametrize("dtype,wdtype", TYPES)
def test_every_width(dtype, wdtype, cols):
    for rows in (1, 3, 37):
        x, w, b, dy = _inputs(rows, cols, dtype, wdtype, seed=cols + rows)
        want, bounds = _reference(x, w, b, dy, 1e-5)
        for got, v, d, what in zip(_run(x, w, b, dy, 1e-5), want, bounds, ("y", "dx", "dw", "db")):
            _check(got, v, d, f"{what} of {rows} x {cols}")


@pytest.mark.parametrize("rows,cols", [(304, 768), (305, 768), (1023, 768), (2432, 64), (5000, 1001), (999, 4096), (700, 8192),
                                       (100, 9000)])
@pytest.mark.parametrize("dtype,wdtype", TYPES)
def test_many_rows(dtype, wdtype, rows, cols):
    x, w, b, dy = _inputs(rows, cols, dtype, wdtype, seed=rows)
    want, bounds = _reference(x, w, b, dy, 1e-6)
    got = _run(x, w, b, dy, 1e-6)
    for g, v, d, what in zip(got, want, bounds, ("y", "dx", "dw", "db")):
        _check(g, v, d, what)
    for first, second in zip(got, _run(x, w, b, dy, 1e-6)):
        assert torch.equal(first, second)


@pytest.mark.parametrize("dtype,wdtype", TYPES)
def test_a_mean_far_from_zero_costs_what_the_inputs_bits_cost(dtype, wdtype):
    x, w, b, dy = _inputs(64, 768, dtype, wdtype, mean=1000.0)
    want, bounds = _reference(x, w, b, dy, 1e-5)
    for g, v, d in zip(_run(x, w, b, dy, 1e-5), want, bounds):
        _check(g, v, d, "far from 0")


def _views(t, kind):
    rows, cols = t.shape
    if kind == "padded":  # rows further apart
        return torch.empty(rows, cols + 24, dtype=t.dtype, device="cuda")[:, 8:8 + cols].copy_(t)
    if kind == "off":  # and off every boundary
        return torch.empty(rows * cols + 1, dtype=t.dtype, device="cuda")[1:].view(rows, cols).copy_(t)
    if kind == "columns":
        return t.t().contiguous().t()
    return t


@pytest.mark.parametrize("cols", [64, 768, 1536, 8200])
@pytest.mark.parametrize("dtype,wdtype", TYPES)
def test_strides_and_alignment(dtype, wdtype, cols):
    x, w, b, dy = _inputs(21, cols, dtype, wdtype)
    want, bounds = _reference(x, w, b, dy, 1e-5)
    for kinds in (("padded", "padded"), ("off", "plain"), ("plain", "off"), ("columns", "plain"), ("plain", "columns")):
        wo = torch.empty(cols + 1, dtype=w.dtype, device="cuda")[1:].copy_(w) if kinds[0] == "off" else w
        got = _run(_views(x, kinds[0]), wo, b, _views(dy, kinds[1]), 1e-5)
        for g, v, d, what in zip(got, want, bounds, ("y", "dx", "dw", "db")):
            _check(g, v, d, f"{what} {kinds}")


def test_without_weight_or_bias():
    x, w, b, dy = _inputs(33, 768, BF16, F32)
    one, zero = torch.ones_like(w), torch.zeros_like(b)
    for weight, bias in ((w, None), (None, b), (None, None)):
        want, bounds = _reference(x, one if weight is None else w, zero if bias is None else b, dy, 1e-5)
        leaves = [x.detach().requires_grad_()] + [t.detach().requires_grad_() for t in (weight, bias) if t is not None]
        y = layer_norm(leaves[0], leaves[1] if weight is not None else None, leaves[-1] if bias is not None else None)
        got = torch.autograd.grad(y, leaves, dy)
        _check(y.detach(), want[0], bounds[0], "y")
        _check(got[0], want[1], bounds[1], "dx")
        if weight is not None:
            _check(got[1], want[2], bounds[2], "dw")
        if bias is not None:
            _check(got[-1], want[3], bounds[3], "db")


def test_shapes_of_more_and_fewer_dimensions_and_of_nothing():
    x, w, b, dy = _inputs(24, 96, BF16, F32)
    flat = _run(x, w, b, dy, 1e-5)
    for shape in ((2, 3, 4, 96), (1, 24, 96)):
        got = _run(x.view(shape), w, b, dy.view(shape), 1e-5)
        assert got[0].shape == got[1].shape == torch.Size(shape)
        for g, f in zip(got, flat):
            assert torch.equal(g.reshape(f.shape), f)
    single = _run(x[5], w, b, dy[5], 1e-5)
    assert torch.equal(single[1], _run(x[5:6], w, b, dy[5:6], 1e-5)[1][0])
    for shape in ((0, 96), (3, 0, 96)):
        y, dx, dw, db = _run(x.new_empty(shape), w, b, x.new_empty(shape), 1e-5)
        assert y.shape == dx.shape == torch.Size(shape)
        assert not dw.any() and not db.any() and dw.shape == w.shape
    y = layer_norm(x.new_empty(4, 0).requires_grad_(), w[:0], b[:0])
    assert y.shape == (4, 0)
    y.sum().backward()


@pytest.mark.parametrize("cols", [200, 768, 4096, 9000])
def test_rows_that_are_not_finite_stay_among_themselves(cols):
    x, w, b, dy = _inputs(40, cols, BF16, BF16)
    clean = _run(x, w, b, dy, 1e-5)
    spoilt = x.clone()
    spoilt[3, 5], spoilt[17, cols - 1], spoilt[39, 0] = float("nan"), float("inf"), float("-inf")
    got = _run(spoilt, w, b, dy, 1e-5)
    bad = torch.zeros(40, dtype=torch.bool, device="cuda")
    bad[[3, 17, 39]] = True
    for g, c in zip(got[:2], clean[:2]):
        assert torch.equal(g[~bad], c[~bad]) and bool(g[bad].isnan().any(1).all())
    assert torch.equal(got[3], clean[3])


def test_columns_that_are_not_there_add_nothing():
    """Whatever they would have: a row of 16 equal values has n = 0, where (0 - 1e30) rstd overflows."""
    x = torch.full((2, 16), 1e30, device="cuda", requires_grad=True)
    w = torch.ones(16, device="cuda", requires_grad=True)
    dy = torch.arange(32, device="cuda").float().view(2, 16)
    dx, dw = torch.autograd.grad(layer_norm(x, w, eps=1e-20), (x, w), dy)
    want = (dy.double() - dy.double().mean(1, keepdim=True)) * 1e10  # rstd = 1 / sqrt(eps), eps within 2^-24 of itself
    assert torch.allclose(dx.double(), want, rtol=2.0 ** -22, atol=0) and not dw.any()


def test_the_gradient_against_differences():
    """Along a random direction h, for f = sum of y dy: (f(x + e h) - f(x - e h)) / 2 e with e = 2^-6.  With |h| of about 1 a
    value the cubic term is of the order e^2 of f's derivative's addends, 2.5e-4, and rounding K U / e of them, 2.3e-4; their
    sum in root mean square over 4 x 513 values is far below 2e-2 of the addends' norm."""
    x, w, b, dy = _inputs(4, 513, F32, F32, seed=3)
    x = x / x.std(1, keepdim=True)
    h = torch.randn_like(x)
    dx, dw, db = _run(x, w, b, dy, 1e-5)[1:]
    e = 2.0 ** -6
    f = lambda x, w=w, b=b: float((layer_norm(x, w, b).double() * dy.double()).sum())
    assert abs((f(x + e * h) - f(x - e * h)) / (2 * e) - float((dx.double() * h).sum())) < 2e-2 * float((dx * h).norm())
    hw = torch.randn_like(w)
    for grad, moved in ((dw, lambda s: f(x, w + s * hw)), (db, lambda s: f(x, w, b + s * hw))):  # linear in both
        assert abs((moved(1.0) - moved(-1.0)) / 2 - float((grad.double() * hw).sum())) < 1e-3 * float((grad * hw).norm())


# ---------------------------------------------------------------------------
# In torch's graph
# ---------------------------------------------------------------------------
def _leaves(rows=24, cols=96, dtype=BF16, wdtype=F32, seed=0):
    x, w, b, dy = _inputs(rows, cols, dtype, wdtype, seed)
    return x.requires_grad_(), w.requires_grad_(), b.requires_grad_(), dy


def test_only_what_is_asked_for():
    x, w, b, dy = _leaves()
    all_of = torch.autograd.grad(layer_norm(x, w, b), (x, w, b), dy)
    for i, leaf in enumerate((x, w, b)):
        assert torch.equal(torch.autograd.grad(layer_norm(x, w, b), leaf, dy)[0], all_of[i])
    for needs in ((True, False, False), (False, True, False), (False, False, True), (False, True, True)):
        leaves = [t.detach().requires_grad_(n) for t, n in zip((x, w, b), needs)]
        layer_norm(*leaves).backward(dy)
        for leaf, n, g in zip(leaves, needs, all_of):
            assert torch.equal(leaf.grad, g) if n else leaf.grad is None
    with torch.no_grad():
        assert not layer_norm(x, w, b).requires_grad


def test_gradients_of_tensors_used_twice_add_up():
    x, w, b, dy = _leaves()
    y = layer_norm(layer_norm(x, w, b), w, b)
    y.backward(dy)
    inner = layer_norm(x.detach(), w.detach(), b.detach()).requires_grad_()
    w2, b2 = w.detach().requires_grad_(), b.detach().requires_grad_()
    d_inner, dw2, db2 = torch.autograd.grad(layer_norm(inner, w2, b2), (inner, w2, b2), dy)
    dx, dw1, db1 = torch.autograd.grad(layer_norm(x, w2, b2), (x, w2, b2), d_inner)
    assert torch.equal(x.grad, dx) and torch.equal(w.grad, dw1 + dw2) and torch.equal(b.grad, db1 + db2)


def test_refusals():
    x, w, b, dy = _leaves()
    for call, match in ((lambda: layer_norm(x, w[:-1], b), "weight"), (lambda: layer_norm(x, w, b[:, None]), "bias"),
                        (lambda: layer_norm(x, w.double(), b), "weight"), (lambda: layer_norm(x, w.cpu(), b), "weight"),
                        (lambda: layer_norm(x, w, b.to(BF16)), "type"), (lambda: layer_norm(x.float(), w.to(BF16)), "weight"),
                        (lambda: layer_norm(x.half()), "float32"), (lambda: layer_norm(x.sum()), "CUDA")):
        with pytest.raises(ValueError, match=match):
            call()
    for eps in (-1e-9, float("nan"), float("inf")):
        with pytest.raises(RuntimeError, match="eps"):
            layer_norm(x, w, b, eps=eps)
    y = layer_norm(x, w, b)
    with pytest.raises(RuntimeError, match="once"):
        torch.autograd.grad(y, x, dy, create_graph=True)
    y.backward(dy)
    with pytest.raises(RuntimeError, match="second time"):
        y.backward(dy)
    with torch.autograd.forward_ad.dual_level():
        for i in range(3):
            args = [t.detach() for t in (x, w, b)]
            args[i] = torch.autograd.forward_ad.make_dual(args[i], torch.ones_like(args[i]))
            with pytest.raises(RuntimeError, match="forward-mode"):
                layer_norm(*args)


def test_inputs_written_to_between_the_passes_are_noticed():
    for which in (0, 1):
        x, w, b, dy = _leaves()
        held = [x * 1, w * 1]
        y = layer_norm(held[0], held[1], b)
        held[which].mul_(2)
        with pytest.raises(RuntimeError, match="modified by an inplace"):
            y.backward(dy)


def test_saved_tensor_hooks():
    x, w, b, dy = _leaves(40, 768)
    want = torch.autograd.grad(layer_norm(x, w, b), (x, w, b), dy)
    with torch.autograd.graph.save_on_cpu():
        y = layer_norm(x, w, b)
    for _ in range(2):
        assert all(torch.equal(a, c) for a, c in zip(torch.autograd.grad(y, (x, w, b), dy, retain_graph=True), want))
    for other in (lambda t: t[:-1], lambda t: t.cpu(), lambda t: t.to(torch.float64)):
        with torch.autograd.graph.saved_tensors_hooks(lambda t: t, other):
            y = layer_norm(x, w, b)
        with pytest.raises(RuntimeError, match="hook"):
            torch.autograd.grad(y, (x, w, b), dy)
    got = torch.utils.checkpoint.checkpoint(lambda t: layer_norm(t, w, b), x, use_reentrant=False)
    assert all(torch.equal(a, c) for a, c in zip(torch.autograd.grad(got, (x, w, b), dy), want))


def test_on_another_stream():
    x, w, b, dy = _leaves(2000, 768)
    want = _run(x, w, b, dy, 1e-5)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y = layer_norm(x, w, b)
        got = (y.detach(), *torch.autograd.grad(y, (x, w, b), dy))
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, c) for a, c in zip(got, want))


def test_captured_and_replayed():
    x, w, b, dy = _leaves(500, 768)
    want = _run(x, w, b, dy, 1e-5)
    eager = layer_norm(x, w, b)  # a graph of the same leaves that lives on meanwhile
    static = [t.detach().clone().requires_grad_() for t in (x, w, b)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.autograd.grad(layer_norm(*static), static, dy)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = layer_norm(*static)
        grads = torch.autograd.grad(y, static, dy)
    with torch.no_grad():
        static[0].mul_(2)
    graph.replay()
    with torch.no_grad():
        static[0].copy_(x)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, c) for a, c in zip((y.detach(), *grads), want))
    assert all(torch.equal(a, c) for a, c in zip(torch.autograd.grad(eager, (x, w, b), dy), want[1:]))


@pytest.mark.parametrize("rows,cols", [(19999, 264), (20003, 511), (20000, 768), (19500, 1000), (14700, 1001), (3100, 2048), (2500, 2056),
                                       (1217, 4096), (1300, 4097), (1300, 5632), (609, 8192)])
@pytest.mark.parametrize("dtype,wdtype", TYPES)
def test_rows_that_a_block_takes_in_turn(dtype, wdtype, rows, cols):
    """Rows on their way ahead of the one that is worked on, more of them than blocks; the last ones ragged; rows apart."""
    x, w, b, dy = _inputs(rows, cols, dtype, wdtype, seed=rows + cols)
    want, bounds = _reference(x, w, b, dy, 1e-5)
    got = _run(_views(x, "padded"), w, b, dy, 1e-5)
    for g, v, d, what in zip(got, want, bounds, ("y", "dx", "dw", "db")):
        _check(g, v, d, what)
    for first, second in zip(got, _run(_views(x, "padded"), w, b, dy, 1e-5)):
        assert torch.equal(first, second)


def test_offsets_past_32_bits():
    """The last rows of more than 2^31 values are as they are alone, but for the order of their sums."""
    rows, cols = 530000, 4096
    x = torch.zeros(rows, cols, dtype=BF16, device="cuda")
    dy = torch.zeros(rows, cols, dtype=BF16, device="cuda")
    assert x.numel() > 2 ** 31
    tail, w, b, dtail = _inputs(100, cols, BF16, F32)
    x[-100:], dy[-100:] = tail, dtail
    want, bounds = _reference(tail, w, b, dtail, 1e-5)
    y, dx, dw, db = _run(x, w, b, dy, 1e-5)
    for g, v, d, what in zip((y[-100:], dx[-100:], dw, db), want, bounds, ("y", "dx", "dw", "db")):
        _check(g, v, d, what)  # (rows of zeros add nothing: dy is 0 there)
    assert not bool(dx[:-100].any()) and torch.equal(y[0], b.bfloat16())


def test_gradients_that_are_broadcast():
    """y.sum() hands back one value with strides of 0, a mean over rows one row; an expanded x is read as what it shows."""
    x, w, b, dy = _inputs(40, 768, F32, F32)
    one_dy = dy[0]
    for make, dy in ((lambda y: y.sum(), torch.ones_like(x)), (lambda y: (y.sum(0) * one_dy).sum(), one_dy.expand_as(x).clone())):
        leaves = [t.clone().requires_grad_() for t in (x, w, b)]
        make(layer_norm(*leaves)).backward()
        want, bounds = _reference(x, w, b, dy, 1e-5)
        for leaf, v, d, what in zip(leaves, want[1:], bounds[1:], ("dx", "dw", "db")):
            _check(leaf.grad, v, d, what)
    one = x[:1]
    assert torch.equal(layer_norm(one.expand(40, 768), w, b), layer_norm(one.repeat(40, 1), w, b))
