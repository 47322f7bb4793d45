"""Orthogonalisation by Newton-Schulz steps and the Muon step against their formulas in 64 bits: wide, tall and square
matrices from a single element to several tiles, odd sizes, strides and alignment of lists, types, values at the ends of
binary32's range; the momentum and the weights' rounding bit for bit."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2607_10611_gb300 import Muon, Orthogonalizer  # noqa: E402

BF16, F32 = torch.bfloat16, torch.float32
TYPES = {"bf16": BF16, "f32": F32}
ABC = (3.4445, -4.7750, 2.0315)
# Products take FP16 values, each off by at most 2^-11 of itself.  The same roundings done in 64 bits leave a relative error in
# the 2-norm of 1.2e-3 to 1.5e-3 after five steps of a random matrix, and less where a few directions dominate (X's second
# part); twice the largest of them:
FAR = 3e-3
# ... where many singular values' errors average out.  A single one's has no such average: it is a weighted sum of about 20
# roundings (X twice, A and B in each step).  A rounding is at most sqrt(3) times its root mean square, and a sum of 20
# terms at most sqrt(20) times the root of the sum of their squares: sqrt(60) times 1.5e-3 in all.
FAR_ALONE = 1.2e-2
SHAPES = [(1, 1), (1, 7), (5, 1), (3, 300), (64, 64), (65, 63), (100, 256), (256, 256), (257, 255), (300, 700), (700, 300), (512, 513),
          (255, 1300), (768, 2304), (1000, 1000)]


def _polar(x, steps=5):
    x = x.double()
    tall = x.shape[0] > x.shape[1]
    x = x.t() if tall else x
    norm = x.norm()
    x = x / norm if norm else x
    a, b, c = ABC
    for _ in range(steps):
        p = x @ x.t()
        x = a * x + (b * p + c * (p @ p)) @ x
    return x.t() if tall else x


def _matrix(rows, cols, dtype=BF16, seed=0, rank=0):
    g = torch.Generator(device="cuda").manual_seed(1000 * rows + cols + seed)
    normal = lambda *s: torch.randn(*s, generator=g, device="cuda")
    x = normal(rows, cols)
    if rank:
        x = normal(rows, rank) @ normal(rank, cols) + 0.05 * x
    return x.to(dtype)


def _near(got, want, far=None):
    half_step = torch.finfo(got.dtype).eps / 2
    assert got.shape == want.shape
    far = far or (FAR if min(got.shape) >= 32 else FAR_ALONE)
    off = float((got.double() - want).norm() / want.norm())
    assert off <= far + half_step, off


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_every_shape(dtype, shape):
    x = _matrix(*shape, TYPES[dtype])
    keep = x.clone()
    ortho = Orthogonalizer([shape], dtype)
    y, = ortho([x])
    assert y.dtype == x.dtype and torch.equal(x, keep)
    _near(y, _polar(x))
    assert torch.equal(ortho([x])[0], y) and ortho.device_status() == 0


@pytest.mark.parametrize("shape", [(300, 700), (700, 300), (512, 512)])
@pytest.mark.parametrize("steps", [1, 2, 3, 4, 6])
def test_other_numbers_of_steps(shape, steps):
    x = _matrix(*shape, F32)
    _near(Orthogonalizer([shape], "f32", steps=steps)([x])[0], _polar(x, steps))


@pytest.mark.parametrize("shape", [(300, 700), (700, 300), (600, 600)])
def test_matrices_that_a_few_directions_dominate(shape):
    """The small singular values' directions too: 64 of rank beside noise of 5 %, most of the result."""
    x = _matrix(*shape, F32, rank=16)
    _near(Orthogonalizer([shape], "f32")([x])[0], _polar(x))


@pytest.mark.parametrize("shape", [(256, 256), (512, 1100), (1100, 512), (700, 700)])
def test_every_element_has_its_place(shape):
    """A permutation's rows, scaled by different powers of two: X stays as sparse, its elements go their own way."""
    rows, cols = shape
    r = min(shape)
    g = torch.Generator(device="cuda").manual_seed(3)
    at = torch.randperm(max(shape), generator=g, device="cuda")[:r]
    x = torch.zeros(shape, device="cuda")
    v = torch.exp2(-(torch.arange(r, device="cuda") % 5).float())
    v[::3] *= -1
    if rows <= cols:
        x[torch.arange(r), at] = v
    else:
        x[at, torch.arange(r)] = v
    y = Orthogonalizer([shape], "f32")([x])[0]
    want = _polar(x)
    assert bool((y[x == 0] == 0).all())
    assert float(((y.double() - want)[x != 0] / want[x != 0]).abs().max()) <= FAR_ALONE


def test_a_list():
    shapes = SHAPES + [(0, 5), (5, 0), (0, 0)] + [(40, 70)] * 3
    for dtype in ("bf16", "f32"):
        xs = [_matrix(r, c, TYPES[dtype], seed=i) for i, (r, c) in enumerate(shapes)]
        ortho = Orthogonalizer(shapes, dtype)
        ys = ortho(xs)
        for x, y, s in zip(xs, ys, shapes):
            assert y.shape == torch.Size(s)
            if x.numel():
                assert torch.equal(y, Orthogonalizer([s], dtype)([x])[0])
        mine = [torch.full_like(x, 7.0) for x in xs]
        back = ortho(xs, out=mine)
        assert all(torch.equal(a, b) for a, b in zip(mine, ys)) and all(a is b for a, b in zip(back, mine))
        ortho(xs, out=xs)  # in place
        assert all(torch.equal(a, b) for a, b in zip(xs, ys))


def test_more_matrices_than_travel_with_a_launch():
    shapes = [(1 + i % 9, 1 + i % 11) for i in range(1000)]
    ortho = Orthogonalizer(shapes, "f32")
    for seed in (0, 1):
        xs = [_matrix(r, c, F32, seed=seed) for r, c in shapes]
        ys = ortho(xs)
        for i in (0, 447, 448, 895, 896, 999):
            _near(ys[i], _polar(xs[i]))
        assert all(torch.equal(a, b) for a, b in zip(ortho(xs), ys))


@pytest.mark.parametrize("offset", [1, 3])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_alignment(dtype, offset):
    for shape in ((48, 64), (64, 48), (33, 65), (200, 311)):
        x = _matrix(*shape, TYPES[dtype])
        want = Orthogonalizer([shape], dtype)([x])[0]
        off = lambda t: torch.empty(t.numel() + offset, dtype=t.dtype, device="cuda")[offset:].view(t.shape).copy_(t)
        out = off(torch.zeros_like(x))
        Orthogonalizer([shape], dtype)([off(x)], out=[out])
        assert torch.equal(out, want)


@pytest.mark.parametrize("power", [-149 + 24, -120, -60, 0, 60, 100, 120])
def test_the_norm_at_the_ends_of_the_range(power):
    """A power of two changes nothing: from values whose squares vanish in binary32 to ones whose squares overflow."""
    shape = (70, 130)
    x = _matrix(*shape, BF16).float().clamp(-4, 4)
    want = Orthogonalizer([shape], "f32")([x])[0]
    scaled = torch.ldexp(x.double(), torch.tensor(power)).float()
    if power > -120:
        assert torch.equal(Orthogonalizer([shape], "f32")([scaled])[0], want)
    _near(Orthogonalizer([shape], "f32")([scaled])[0], _polar(scaled))


def test_the_smallest_numbers():
    x = torch.zeros(8, 8, device="cuda")
    x[0, 0] = 2.0 ** -149
    y = Orthogonalizer([(8, 8)], "f32")([x])[0]
    _near(y, _polar(x))


def test_zeros_and_values_that_are_not_finite():
    shapes = [(20, 30), (30, 20), (20, 30), (300, 30)]
    xs = [_matrix(*s, F32) for s in shapes]
    clean = Orthogonalizer(shapes, "f32")(xs)
    xs[0].zero_()
    xs[1][3, 4] = float("nan")
    xs[2][0, 0] = float("inf")
    ys = Orthogonalizer(shapes, "f32")(xs)
    assert not ys[0].any()
    assert bool(ys[1].isnan().all()) and bool(ys[2].isnan().all())
    assert torch.equal(ys[3], clean[3])


# ---------------------------------------------------------------------------
# The step
# ---------------------------------------------------------------------------
class Reference:
    """The step on copies: momentum and U in binary32 as defined, O in 64 bits."""

    def __init__(self, w, m, **kw):
        self.w, self.m = [t.clone() for t in w], [t.clone() for t in m]
        self.kw = kw

    def step(self, grads, lr, scale=None):
        beta = np.float32(self.kw["momentum"])
        rest = float(np.float32(1.0 - float(beta)))
        beta, lr = float(beta), float(np.float32(lr))
        decay = float(np.float32(lr * float(np.float32(self.kw["weight_decay"]))))
        out, sizes = [], []
        for i, g in enumerate(grads):
            g = g.float() * (1.0 if scale is None else scale)
            m = self.m[i].float() * beta + g * rest
            u = m * beta + g * rest if self.kw["nesterov"] else m
            self.m[i].copy_(m)
            rows, cols = u.shape
            factor = 0.2 * math.sqrt(max(rows, cols)) if self.kw["scale"] == "rms" else math.sqrt(max(1.0, rows / cols))
            o = _polar(u) if u.numel() else u.double()
            out.append(self.w[i].double() * (1 - decay) - lr * factor * o)
            sizes.append(lr * factor * float(o.norm()))
        return out, sizes


def _list(shapes, weights, momentum, grads, seed=0):
    w = [0.02 * _matrix(*s, F32, seed).to(TYPES[weights]) for s in shapes]
    m = [1e-3 * _matrix(*s, F32, seed + 1).to(TYPES[momentum]) for s in shapes]
    g = [1e-3 * _matrix(*s, F32, seed + 2).to(TYPES[grads]) for s in shapes]
    return w, m, g


LIST = [(64, 96), (96, 64), (1, 50), (50, 1), (33, 47), (0, 4), (130, 130), (300, 261), (520, 264)]


@pytest.mark.parametrize("weights,momentum,grads", [("bf16", "f32", "bf16"), ("f32", "f32", "f32"), ("f32", "bf16", "bf16"),
                                                    ("bf16", "bf16", "f32")])
@pytest.mark.parametrize("nesterov,scale", [(True, "rms"), (False, "spectral")])
def test_steps(weights, momentum, grads, nesterov, scale):
    w, m, g = _list(LIST, weights, momentum, grads)
    kw = dict(momentum=0.9, weight_decay=0.1, nesterov=nesterov, scale=scale)
    ref = Reference(w, m, **kw)
    copies = [torch.full(s, 9.0, dtype=BF16, device="cuda") for s in LIST] if weights == "f32" else None
    opt = Muon(w, m, weight_dtype=weights, grad_dtype=grads, momentum_dtype=momentum, compute=copies, **kw)
    for t in range(1, 4):
        ref.w = [x.clone() for x in w]
        scaled = torch.tensor([0.5], device="cuda") if t == 2 else None
        want, sizes = ref.step(g, 0.01, 0.5 if t == 2 else None)
        opt.step(g, t, 0.01, grad_scale=scaled)
        for i, (x, v, size) in enumerate(zip(w, want, sizes)):
            assert torch.equal(m[i], ref.m[i]), (t, i)
            # O's error in the 2-norm, and the weight's rounding of each value
            rounding = float(v.norm()) * torch.finfo(x.dtype).eps / 2
            far = FAR if min(x.shape) >= 32 else FAR_ALONE
            assert float((x.double() - v).norm()) <= far * size + rounding + 4 * 2.0 ** -24 * float(v.norm()), (t, i)
            if copies:
                assert torch.equal(copies[i], x.to(BF16))
    assert opt.device_status() == 0


def _lanes(shapes, seed, t):
    """Each matrix's 16 random bits, by the library's own lanes at the list's global indices."""
    from paper_2607_10611_gb300 import _native as N
    out, first = [], 0
    for r, c in shapes:
        n = r * c
        lanes = torch.zeros(max(1, -(-n // 8) * 8), dtype=torch.int32, device="cuda")
        if n:
            N.mpadam_rng_lanes(seed, t, N.MPADAM_BF16, first, lanes.numel(), lanes.data_ptr(), torch.cuda.current_stream().cuda_stream)
        out.append(lanes[:n].view(r, c))
        first += -(-n // 128) * 128
    return out


@pytest.mark.parametrize("rounding", ["nearest", "stochastic"])
def test_bf16_weights_are_the_binary32_ones_rounded(rounding):
    """Bit for bit: the same step on the same values in binary32 is what is rounded."""
    w, m, g = _list(LIST, "bf16", "f32", "bf16")
    w32, m32 = [x.float() for x in w], [x.clone() for x in m]
    kw = dict(momentum=0.95, weight_decay=0.02, seed=77)
    Muon(w32, m32, weight_dtype="f32", **kw).step(g, 5, 0.02)
    Muon(w, m, weight_dtype="bf16", rounding=rounding, **kw).step(g, 5, 0.02)
    for x, y, bits in zip(w, w32, _lanes(LIST, 77, 5)):
        if rounding == "nearest":
            assert torch.equal(x, y.to(BF16))
        else:
            u = y.view(torch.int32)
            away = (bits & 0xFFFF) < (u & 0xFFFF)
            assert torch.equal(x.view(torch.int16), ((u >> 16) + away.int()).to(torch.int16))


def test_without_decay_or_learning_rate():
    w, m, g = _list(LIST, "f32", "f32", "f32")
    keep = [x.clone() for x in w]
    Muon(w, m, weight_dtype="f32", grad_dtype="f32", weight_decay=0.5).step(g, 1, 0.0)
    assert all(torch.equal(a, b) for a, b in zip(w, keep))


@pytest.mark.parametrize("offset", [1, 2])
def test_lists_off_their_boundaries(offset):
    off = lambda t: torch.empty(t.numel() + offset, dtype=t.dtype, device="cuda")[offset:].view(t.shape).copy_(t)
    for weights, momentum, grads in (("bf16", "bf16", "f32"), ("f32", "f32", "bf16")):
        w, m, g = _list(LIST, weights, momentum, grads)
        w2, m2, g2 = ([off(t) for t in l] for l in (w, m, g))
        for a, b, c in ((w, m, g), (w2, m2, g2)):
            Muon(a, b, weight_dtype=weights, momentum_dtype=momentum, grad_dtype=grads, rounding="stochastic").step(c, 1, 0.01)
        assert all(torch.equal(a, b) for a, b in zip(w + m, w2 + m2))


def test_a_multiplier_that_is_nan_changes_nothing():
    w, m, g = _list(LIST, "bf16", "f32", "bf16")
    keep = [x.clone() for x in w + m]
    opt = Muon(w, m)
    opt.step(g, 1, 0.01, grad_scale=torch.tensor([float("nan")], device="cuda"))
    assert all(torch.equal(a, b) for a, b in zip(w + m, keep))
    opt.step(g, 1, 0.01, grad_scale=torch.tensor([1.0], device="cuda"))
    again = [x.clone() for x in keep]
    Muon(again[:len(w)], again[len(w):]).step(g, 1, 0.01)
    assert all(torch.equal(a, b) for a, b in zip(w + m, again))


def test_momentum_that_fades_keeps_its_direction():
    """A matrix that gets no gradients (an expert that no token reaches): U shrinks below binary32's squares, O stays."""
    w, m, g = _list([(40, 60), (60, 40)], "f32", "f32", "f32")
    m[1].mul_(1e-30)
    g = [torch.zeros_like(x) for x in g]
    u = [x.clone() for x in m]
    before = [x.clone() for x in w]
    Muon(w, m, weight_dtype="f32", grad_dtype="f32", weight_decay=0.0, scale="spectral").step(g, 1, 0.1)
    for x, b, v, s in zip(w, before, u, (1.0, math.sqrt(1.5))):
        _near((b.double() - x.double()) / (0.1 * s), _polar(v), FAR + 1e-4)  # the difference's own roundings


def test_captured_and_replayed_on_another_stream():
    w, m, g = _list(LIST, "f32", "f32", "f32")
    w2, m2 = [x.clone() for x in w], [x.clone() for x in m]
    opt = Muon(w, m, weight_dtype="f32", grad_dtype="f32")
    lr = 0.01
    graph = torch.cuda.CUDAGraph()
    static = [x.clone() for x in g]
    with torch.cuda.graph(graph):
        opt.step(static, 1, lr)
    other = Muon(w2, m2, weight_dtype="f32", grad_dtype="f32")
    side = torch.cuda.Stream()
    for k in range(3):
        for s, x in zip(static, g):
            s.copy_(x * (k + 1))
        graph.replay()
        side.wait_stream(torch.cuda.current_stream())
        now = [x * (k + 1) for x in g]
        side.wait_stream(torch.cuda.current_stream())
        other.step(now, 1, lr, stream=side)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(w + m, w2 + m2))


def test_a_list_larger_than_one_workspace():
    """Matrices that share the workspace one group after another: 16384 x 16384 takes 2.5 GiB."""
    shapes = [(16384, 16384)] * 3 + [(64, 80)]
    small = _matrix(64, 80, BF16)
    xs = [torch.zeros(s, dtype=BF16, device="cuda") for s in shapes[:3]] + [small]
    for k, x in enumerate(xs[:3]):
        x[k, :5] = 1.0
    ys = Orthogonalizer(shapes, "bf16")(xs)
    for k, y in enumerate(ys[:3]):
        want = _polar(xs[k][:k + 1].float())
        assert torch.allclose(y[k, :5].double(), want[k, :5], rtol=FAR_ALONE + 2.0 ** -8, atol=0) and int((y != 0).sum()) == 5
    assert torch.equal(ys[3], Orthogonalizer([(64, 80)], "bf16")([small])[0])


def test_refusals():
    w, m, g = _list([(6, 8), (8, 6)], "bf16", "f32", "bf16")
    opt = Muon(w, m)
    for bad in ([g[0]], [g[0], g[0]], [g[0], g[1].t()], [g[0], g[1].float()], [g[0], g[1].cpu()], [g[0], g[1].view(-1)]):
        with pytest.raises(ValueError):
            opt.step(bad, 1, 0.01)
    for t, lr in ((0, 0.01), (1, -1.0), (1, float("nan"))):
        with pytest.raises(RuntimeError):
            opt.step(g, t, lr)
    with pytest.raises(ValueError):
        opt.step(g, 1, 0.01, grad_scale=torch.ones(1, device="cuda", dtype=torch.float64))
    for args in ((w, m[:1]), (w, [m[0], m[0]]), ([w[0], w[1].t()], m), ([x.float() for x in w], m), (w, [x.to(BF16) for x in m]),
                 ([x.view(-1) for x in w], [x.view(-1) for x in m])):
        with pytest.raises(ValueError):
            Muon(*args)
    with pytest.raises(RuntimeError, match="compute"):
        Muon(w, m, compute=[x.clone() for x in w])
    ortho = Orthogonalizer([(6, 8), (8, 6)])
    for x, out in (([g[0]], None), (g[::-1], None), (g, [g[0]]), (g, g[::-1]), (g, [x.float() for x in g])):
        with pytest.raises(ValueError):
            ortho(x, out=out)
    assert Orthogonalizer([])([]) == [] and Muon([], []).step([], 1, 0.1) is None


@pytest.mark.parametrize("shape", [(1300, 1500), (1537, 1281), (1290, 2600), (2100, 1800)])
def test_several_rows_of_tiles_read_from_below_the_diagonal(shape):
    """Six to eight tiles to a side: most of A and B is read turned."""
    x = _matrix(*shape, F32, rank=40)
    ortho = Orthogonalizer([shape], "f32")
    y, = ortho([x])
    _near(y, _polar(x))
    assert torch.equal(ortho([x])[0], y) and ortho.device_status() == 0


def test_a_mixed_list_gives_what_its_matrices_give_alone():
    """The tiles of large and small, wide and tall matrices are taken in turn, and wait for their own matrix's alone: the
    squares' sums apart, which a matrix's own sizes decide, nothing depends on the list."""
    shapes = [(1400, 300), (1, 1), (900, 900), (17, 2000), (2000, 17), (513, 1025), (256, 512), (3, 3), (700, 1300), (1024, 64)]
    x = [_matrix(*s, F32, seed=i) for i, s in enumerate(shapes)]
    together = Orthogonalizer(shapes, "f32")
    want = together(x)
    for s, m, y in zip(shapes, x, want):
        assert torch.equal(Orthogonalizer([s], "f32")([m])[0], y)
    for _ in range(20):
        assert all(torch.equal(a, b) for a, b in zip(together(x), want))
    assert together.device_status() == 0


def test_two_lists_at_once_on_two_streams():
    """Each with a workspace and counters of its own; their pairs of CTAs share the SMs."""
    lists = [[(1100, 700)] * 6, [(300, 300)] * 40]
    x = [[_matrix(*s, F32, seed=i) for i, s in enumerate(shapes)] for shapes in lists]
    ortho = [Orthogonalizer(shapes, "f32") for shapes in lists]
    want = [o(m) for o, m in zip(ortho, x)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[], []]
    for _ in range(5):
        for i in (0, 1):
            got[i].append(ortho[i](x[i], stream=streams[i]))
    torch.cuda.synchronize()
    for i in (0, 1):
        assert all(torch.equal(a, b) for call in got[i] for a, b in zip(call, want[i])) and ortho[i].device_status() == 0


def test_offsets_past_32_bits():
    """A block in the last corner of zeros comes out as it does alone, in its place."""
    rows, cols, block = 70001, 33001, (300, 400)
    x = torch.zeros(rows, cols, dtype=BF16, device="cuda")
    assert x.numel() > 2 ** 31
    corner = _matrix(*block)
    x[-block[0]:, -block[1]:] = corner
    ortho = Orthogonalizer([(rows, cols)], "bf16")
    y, = ortho([x])
    assert ortho.device_status() == 0
    _near(y[-block[0]:, -block[1]:].clone(), _polar(corner))
    assert not bool(y[:-block[0]].any()) and not bool(y[-block[0]:, :-block[1]].any())


def test_two_graphs_of_one_state_one_after_another():
    """They share the workspace and its counters, and leave them as the next one needs them, an eager call too."""
    shapes = [(600, 900), (300, 100), (1, 5)]
    x = [_matrix(*s, F32, seed=i) for i, s in enumerate(shapes)]
    z = [_matrix(*s, F32, seed=7 + i) for i, s in enumerate(shapes)]
    ortho = Orthogonalizer(shapes, "f32")
    want_x, want_z = ortho(x), ortho(z)
    graphs, outs, stream = [], [], torch.cuda.Stream()
    for v in (x, z):
        out = [torch.zeros_like(t) for t in v]
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g, stream=stream):
            ortho(v, out=out)
        graphs.append(g), outs.append(out)
    for _ in range(3):
        graphs[0].replay()
        graphs[1].replay()
        eager = ortho(x)
        torch.cuda.synchronize()
        for got, want in ((outs[0], want_x), (outs[1], want_z), (eager, want_x)):
            assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert ortho.device_status() == 0
