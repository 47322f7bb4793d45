"""The AdamW step and the gradient norm against plain references: the canonical binary32 sequence bit for bit, and
binary64 within what its roundings allow."""
import ctypes
import math
import subprocess
from pathlib import Path

import numpy as np
import pytest
import torch

import fp8_reference as R

pytestmark = pytest.mark.gpu

from paper_2607_10611_gb300.adamw import AdamW, GradNorm  # noqa: E402

SIZES = [0, 1, 7, 8, 9, 127, 128, 129, 300, 2047, 2048, 2049, 6000, 0, 5]
HP = dict(lr=3e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.1)


class Problem:
    """A list on the GPU and the same in numpy.  offset: elements by which every array starts off its alignment."""

    def __init__(self, sizes, weights, grads, state, seed=0, offset=0, compute=False, special=False):
        self.rng, self.sizes, self.offset = np.random.default_rng(seed), sizes, offset
        self.weights, self.gdtype, self.state, self.special = weights, grads, state, special
        low = state == "e4m3"
        self.w, self.m, self.v, self.ms, self.vs = [], [], [], [], []
        for n in sizes:
            w = (0.02 * self.rng.normal(size=n)).astype(np.float32)
            self.w.append(w if weights == "f32" else R.bf16_value(R.bf16_nearest(w)))
            m = (1e-3 * self.rng.normal(size=n)).astype(np.float32)
            r = (1e-3 * np.abs(self.rng.normal(size=n))).astype(np.float32)
            if special and n > 128:  # a block that never saw a gradient, and one with a huge spread
                m[:128] = r[:128] = 0.0
                r[128:256] *= np.exp2(self.rng.uniform(-30, 0, r[128:256].size)).astype(np.float32)
            if low:
                for x, codes, scales, keep in ((m, self.m, self.ms, False), (r, self.v, self.vs, True)):
                    c, s = R.encode_blocks(x, None, keep) if n else (np.zeros(0, np.uint8), np.zeros(0, np.uint8))
                    codes.append(c)
                    scales.append(s)
            else:
                self.m.append(m)
                self.v.append(r * r)
        put = self.put
        wd = torch.float32 if weights == "f32" else torch.bfloat16
        self.gw = [put(x, wd) for x in self.w]
        if low:
            self.gm, self.gv = ([put(x, torch.uint8).view(torch.float8_e4m3fn) for x in y] for y in (self.m, self.v))
            self.gms, self.gvs = ([put(x, torch.uint8).view(torch.float8_e8m0fnu) for x in y] for y in (self.ms, self.vs))
        else:
            self.gm, self.gv = ([put(x, torch.float32) for x in y] for y in (self.m, self.v))
        self.gc = [put(np.zeros(n, np.float32), torch.bfloat16) for n in sizes] if compute else None

    def put(self, x, dtype):
        store = torch.zeros(len(x) + self.offset, dtype=dtype, device="cuda")
        view = store[self.offset:]
        view.copy_(torch.from_numpy(np.ascontiguousarray(x)))
        return view

    def grads(self):
        out = []
        for n in self.sizes:
            g = (1e-3 * self.rng.normal(size=n)).astype(np.float32)
            if self.special and n > 128:
                g[:128] = 0.0
                g[130::7] = 0.0
            out.append(g if self.gdtype == "f32" else R.bf16_value(R.bf16_nearest(g)))
        dt = torch.float32 if self.gdtype == "f32" else torch.bfloat16
        return out, [self.put(g, dt) for g in out]

    def optimizer(self, **kw):
        hp = {k: v for k, v in HP.items() if k != "lr"}
        low = dict(m_scales=self.gms, v_scales=self.gvs) if self.state == "e4m3" else {}
        self.opt = AdamW(self.gw, self.gm, self.gv, weight_dtype=self.weights, grad_dtype=self.gdtype,
                         state_dtype=self.state, compute=self.gc, **low, **{**hp, **kw})
        return self.opt

    def reference_step(self, grads, t, seed, rounding, state_rounding, mult=None, hp=HP):
        goff = 0
        for i, n in enumerate(self.sizes):
            if n:
                low = self.state == "e4m3"
                m, v = self.m[i], self.v[i]
                if low:
                    m = R.decode_blocks(m, self.ms[i])
                    r = R.decode_blocks(v, self.vs[i])
                    v = r * r
                w, m, r, v = R.adamw(self.w[i], grads[i], m, v, t=t, mult=mult, **hp)
                if low:
                    lm, lr = R.state_lanes(goff, n, t, seed) if state_rounding == "stochastic" else (None, None)
                    self.m[i], self.ms[i] = R.encode_blocks(m, lm, False)
                    self.v[i], self.vs[i] = R.encode_blocks(r, lr, True)
                else:
                    self.m[i], self.v[i] = m, v
                if self.weights == "f32":
                    self.w[i] = w
                elif rounding == "stochastic":
                    self.w[i] = R.bf16_value(R.bf16_stochastic(w, R.weight_lanes(goff, n, t, seed)))
                else:
                    self.w[i] = R.bf16_value(R.bf16_nearest(w))
            goff += -(-n // 128) * 128

    def check(self):
        if hasattr(self, "opt"):
            assert self.opt.device_status() == 0
        for i, n in enumerate(self.sizes):
            def same(t, want):
                got = t.cpu()
                got = got.view(torch.uint8).numpy() if got.element_size() == 1 else got.float().numpy()
                np.testing.assert_array_equal(got, want, err_msg=f"tensor {i} of {n}")
            same(self.gw[i], self.w[i])
            same(self.gm[i], self.m[i])
            same(self.gv[i], self.v[i])
            if self.state == "e4m3":
                same(self.gms[i], self.ms[i])
                same(self.gvs[i], self.vs[i])
            if self.gc:
                same(self.gc[i], R.bf16_value(R.bf16_nearest(self.w[i])))


@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("grads", ["f32", "bf16"])
@pytest.mark.parametrize("weights,rounding,state,state_rounding", [
    ("f32", "nearest", "f32", "nearest"), ("bf16", "nearest", "f32", "nearest"), ("bf16", "stochastic", "f32", "nearest"),
    ("f32", "stochastic", "f32", "nearest"), ("f32", "stochastic", "e4m3", "stochastic"),  # (a BF16 weight's rounding)
    ("f32", "nearest", "e4m3", "nearest"), ("f32", "nearest", "e4m3", "stochastic"), ("bf16", "nearest", "e4m3", "nearest"),
    ("bf16", "stochastic", "e4m3", "nearest"), ("bf16", "nearest", "e4m3", "stochastic"),
    ("bf16", "stochastic", "e4m3", "stochastic")])
def test_steps_bit_for_bit(weights, rounding, state, state_rounding, grads, offset):
    p = Problem(SIZES, weights, grads, state, offset=offset, compute=weights == "f32", special=True)
    seed = 0x123456789ABCDEF
    opt = p.optimizer(rounding=rounding, state_rounding=state_rounding, seed=seed)
    mult = np.float32(0.37)
    for t in (1, 2, 1000):
        host, dev = p.grads()
        use = t != 2
        opt.step(dev, t, HP["lr"], grad_scale=torch.tensor([mult], device="cuda") if use else None)
        p.reference_step(host, t, seed, rounding, state_rounding, mult if use else None)
        p.check()


def test_many_tiles_and_steps_beyond_32_bits():
    p = Problem([700001, 3, 1 << 20], "bf16", "bf16", "e4m3", seed=3)
    opt = p.optimizer(rounding="stochastic", seed=5)
    t = (1 << 33) + 7
    host, dev = p.grads()
    opt.step(dev, t, HP["lr"])
    p.reference_step(host, t, 5, "stochastic", "stochastic")
    p.check()


@pytest.mark.parametrize("weights", ["bf16", "f32"])
@pytest.mark.parametrize("kw", [dict(), dict(eps=1e-30), dict(eps=1e-33), dict(eps=1e7), dict(beta1=0.0), dict(beta2=0.0),
                                dict(beta2=0.9999999), dict(weight_decay=0.0), dict(lr=0.0)])
def test_every_range_bit_for_bit(kw, weights):
    """Gradients and moments from subnormal to beyond where squares overflow, by blocks and within them: the step's common
    path, what it leaves to the general code, and every border between the two."""
    hp = {**HP, **kw}
    p = Problem([128 * 40, 3000], weights, "f32", "e4m3", seed=11)
    opt = p.optimizer(rounding="stochastic" if weights == "bf16" else "nearest", seed=9, **{k: v for k, v in hp.items() if k != "lr"})
    for t in (1, 2, 3, 500):
        host, dev = p.grads()
        for i, n in enumerate(p.sizes):
            scale = np.exp2(p.rng.uniform(-45, 30, -(-n // 128))).repeat(128)[:n]
            scale[::131] *= np.exp2(p.rng.uniform(-90, 50, scale[::131].size))
            with np.errstate(over="ignore", under="ignore"):
                host[i] = (host[i] * scale).astype(np.float32)
            host[i][5::17] = 0.0
            dev[i].copy_(torch.from_numpy(host[i]))
        opt.step(dev, t, hp["lr"])
        p.reference_step(host, t, 9, "stochastic" if weights == "bf16" else "nearest", "stochastic", hp=hp)
        p.check()


@pytest.mark.parametrize("weights", ["bf16", "f32"])
@pytest.mark.parametrize("kw", [dict(weight_decay=0.0), dict(), dict(eps=1.0), dict(eps=1e-30, weight_decay=0.0), dict(lr=0.0)])
def test_small_weights_beside_small_moments_bit_for_bit(kw, weights):
    """Zeros of either sign, subnormal and small weights, each beside gradients and moments that are zero, subnormal or
    small: the quotient's tiny results, and the sign of what they leave."""
    hp = {**HP, **kw}
    p = Problem([256 * 60, 1000], weights, "f32", "e4m3", seed=12)
    for i, n in enumerate(p.sizes):
        w = np.exp2(p.rng.uniform(-150, 2, n)).astype(np.float32) * np.where(p.rng.random(n) < 0.5, -1, 1).astype(np.float32)
        w[p.rng.random(n) < 0.2] = 0.0
        w[p.rng.random(n) < 0.2] = -0.0
        w[256 * 3:256 * 5] = np.float32(0.5)  # parts without a small weight
        p.w[i] = w if weights == "f32" else R.bf16_value(R.bf16_nearest(w))
        p.gw[i].copy_(torch.from_numpy(p.w[i]))
        for codes, gpu in ((p.m[i], p.gm[i]), (p.v[i], p.gv[i])):
            codes[p.rng.random(n) < 0.3] = 0
            gpu.view(torch.uint8).copy_(torch.from_numpy(codes))
    opt = p.optimizer(rounding="nearest", seed=9, **{k: v for k, v in hp.items() if k != "lr"})
    for t in (1, 2, 3):
        host, dev = p.grads()
        for i, n in enumerate(p.sizes):
            g = host[i] * np.exp2(p.rng.uniform(-130, 0, n)).astype(np.float32)
            g[p.rng.random(n) < 0.3] = 0.0
            host[i] = g
            dev[i].copy_(torch.from_numpy(g))
        opt.step(dev, t, hp["lr"])
        p.reference_step(host, t, 9, "nearest", "stochastic", hp=hp)
        p.check()
        for gpu, w in zip(p.gw, p.w):
            np.testing.assert_array_equal(np.signbit(gpu.float().cpu().numpy()), np.signbit(w))


@pytest.mark.parametrize("decay", [0.0, 0.3])
def test_update_in_64_bits(decay):
    """u = lr m^ / (sqrt(v^) + eps) from nine roundings of binary32 (five of them under the root or in m with at most a
    factor two of cancellation, since both moments' terms are taken of one sign): 16 units of 2^-24 of |u| and 3 of |w|."""
    g = np.random.default_rng(1)
    n = 5000
    w = g.normal(size=n).astype(np.float32)
    gr, m = (np.abs(g.normal(size=n)).astype(np.float32) for _ in range(2))
    v = np.square(g.normal(size=n)).astype(np.float32) + np.float32(1e-3)
    hp = dict(HP, weight_decay=decay)
    put = lambda x: torch.from_numpy(x.copy()).cuda()
    tw, tm, tv = put(w), put(m), put(v)
    opt = AdamW([tw], [tm], [tv], weight_dtype="f32", grad_dtype="f32", **{k: x for k, x in hp.items() if k != "lr"})
    opt.step([put(gr)], 7, hp["lr"])
    ew, em, _, ev = R.adamw(w, gr, m, v, t=7, dtype=np.float64, **hp)
    # betas and 1 - beta are binary32 on both sides: the reference in 64 bits rounds only 1 - beta less
    assert np.all(np.abs(tm.cpu().numpy() - em) <= 4 * 2.0 ** -24 * np.abs(em))
    assert np.all(np.abs(tv.cpu().numpy() - ev) <= 5 * 2.0 ** -24 * np.abs(ev))
    assert np.all(np.abs(tw.cpu().numpy() - ew) <= 2.0 ** -24 * (3 * (np.abs(w) + np.abs(ew)) + 16 * np.abs(ew - w)))


def test_a_root_above_zero_never_becomes_zero():
    """One large second moment beside small ones: their codes underflow, and stay at the smallest code."""
    n = 128
    w = torch.zeros(n, device="cuda")
    st = AdamW.init_state([w])
    g = torch.full((n,), 1e-9, device="cuda")
    g[5] = 1e3
    opt = AdamW([w], st.pop("m"), st.pop("v"), weight_dtype="f32", grad_dtype="f32", **st, weight_decay=0.0)
    opt.step([g], 1, 1e-3)
    codes = opt.v[0].view(torch.uint8)
    assert int(codes.min()) == 1
    assert bool((w.abs() <= 1.001e-3).all())  # this step divides by the root before it is rounded
    opt.step([torch.zeros_like(g)], 2, 1e-3)
    assert bool(torch.isfinite(w).all()) and float(w.abs().max()) < 2.1e-3


def test_stochastic_states_follow_a_slow_average():
    """beta2 = 0.999: nearest codes of the root stand still, stochastic ones follow.  The root is rounded without bias,
    its square is not: a step by d of the root adds d times the grid's spacing to it, at most 1/16 of what the step adds
    itself.  The spread of 4096 elements' mean is below 0.02."""
    n, steps = 4096, 400
    paths = {}
    for rounding in ("nearest", "stochastic"):
        w = torch.zeros(n, device="cuda")
        st = AdamW.init_state([w])
        opt = AdamW([w], st.pop("m"), st.pop("v"), weight_dtype="f32", grad_dtype="f32", state_rounding=rounding, **st)
        opt.step([torch.ones(n, device="cuda")], 1, 0.0)
        for t in range(2, steps):
            opt.step([torch.full((n,), 2.0, device="cuda")], t, 0.0)
        s = opt.v_scales[0].float().repeat_interleave(128)
        paths[rounding] = float((opt.v[0].float() * s).square().mean())
    v = 0.001
    for _ in range(2, steps):
        v = 0.999 * v + 0.004
    assert abs(paths["stochastic"] / v - 1) < 1 / 16 + 0.02
    assert abs(paths["nearest"] / v - 1) > 0.5


def test_a_step_with_a_norm_that_is_not_finite_changes_nothing():
    p = Problem([300, 2049], "bf16", "bf16", "e4m3")
    opt = p.optimizer(rounding="stochastic")
    _, dev = p.grads()
    dev[1][17] = float("inf")
    norm = GradNorm(p.sizes, "bf16")
    out = norm(dev, 1.0)
    assert math.isinf(float(out[0])) and math.isnan(float(out[1]))
    opt.step(dev, 1, 1e-3, grad_scale=out[1:])
    p.check()


def test_not_finite_gradients_without_a_multiplier_stay_in_their_elements():
    p = Problem([300], "f32", "f32", "e4m3")
    opt = p.optimizer(state_rounding="nearest")
    host, dev = p.grads()
    for i, x in ((3, np.nan), (150, np.inf), (151, -np.inf)):
        host[0][i] = x
        dev[0][i] = float(x)
    opt.step(dev, 1, HP["lr"])
    p.reference_step(host, 1, 0, "nearest", "nearest")
    p.check()


@pytest.mark.parametrize("n", [448, 449, 1000])
def test_long_lists_and_changing_gradients(n):
    sizes = [1 + i % 300 for i in range(n)]
    p = Problem(sizes, "f32", "f32", "f32", seed=n)
    opt = p.optimizer()
    norm = GradNorm(sizes, "f32")
    keep = []
    for t in range(1, 4):
        host, dev = p.grads()
        keep.append(dev)  # the next step's gradients lie elsewhere
        opt.step(dev, t, HP["lr"])
        p.reference_step(host, t, 0, "nearest", "nearest")
        want = math.sqrt(sum(float(np.square(x.astype(np.float64)).sum()) for x in host))
        assert abs(float(norm(dev)[0]) / want - 1) < 1e-6
    p.check()


@pytest.mark.parametrize("n", [3, 500])
def test_captured_steps_replay(n):
    sizes = [257] * n
    p = Problem(sizes, "f32", "f32", "f32")
    opt, norm = p.optimizer(), GradNorm(sizes, "f32")
    host, dev = p.grads()
    other_host, other = p.grads()
    out = torch.zeros(2, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        norm(dev, 0.01, out=out)
        opt.step(dev, 5, HP["lr"], grad_scale=out[1:])

    def expect(g, t):
        want = np.sqrt(sum(np.square(x.astype(np.float64)).sum() for x in g))
        assert abs(float(out[0]) / want - 1) < 1e-6
        p.reference_step(g, t, 0, "nearest", "nearest", np.float32(float(out[1])))
        p.check()

    graph.replay()
    expect(host, 5)
    norm(other, 0.01, out=out)
    opt.step(other, 6, HP["lr"], grad_scale=out[1:])
    expect(other_host, 6)
    graph.replay()
    expect(host, 5)
    norm(other, 0.01, out=out)
    opt.step(other, 7, HP["lr"], grad_scale=out[1:])
    expect(other_host, 7)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sizes", [[], [0], [1], [5, 0, 2048, 2049], [3000001, 17, 100]])
def test_norm(sizes, dtype):
    """Within a thread at most 2000 squares are added in binary32 (here far fewer), so the sum of squares is within
    2000 2^-24 of itself and the norm within half of that."""
    g = np.random.default_rng(2)
    td = torch.float32 if dtype == "f32" else torch.bfloat16
    x = [torch.from_numpy(g.normal(size=n)).to(td) for n in sizes]
    want = math.sqrt(sum(float(t.double().square().sum()) for t in x))
    norm = GradNorm(sizes, dtype)
    dev = [t.cuda() for t in x]
    a = norm(dev, 2.0).cpu()
    assert abs(float(a[0]) - want) <= 1000 * 2.0 ** -24 * want
    mult = min(1.0, 2.0 / want) if want else 1.0
    assert abs(float(a[1]) - mult) <= 1001 * 2.0 ** -24 * mult
    assert float(norm(dev)[1]) == 1.0
    for _ in range(3):
        assert torch.equal(norm(dev, 2.0).cpu(), a)  # the same bits every time
    shifted = []
    for t in dev:  # and where every gradient is off its alignment
        s = torch.zeros(t.numel() + 1, dtype=td, device="cuda")
        s[1:] = t
        shifted.append(s[1:])
    assert torch.equal(norm(shifted, 2.0).cpu(), a)


def test_norm_of_what_is_not_finite():
    x = torch.ones(5000, device="cuda")
    norm = GradNorm([5000], "f32")
    for bad, test in ((math.nan, math.isnan), (math.inf, math.isinf), (1e30, math.isinf)):
        x[4999] = bad
        out = norm([x], 1.0).cpu()
        assert test(float(out[0])) and math.isnan(float(out[1]))
    x[4999] = 1.0
    assert float(norm([x], 1.0)[0]) == pytest.approx(math.sqrt(5000.0), rel=1e-6)


def test_other_streams():
    p = Problem([5000, 12], "f32", "f32", "f32")
    opt = p.optimizer()
    host, dev = p.grads()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    opt.step(dev, 1, HP["lr"], stream=side)
    with torch.cuda.stream(side):
        opt.step(dev, 2, HP["lr"])
    side.synchronize()
    for t in (1, 2):
        p.reference_step(host, t, 0, "nearest", "nearest")
    p.check()


def test_refusals():
    w = torch.zeros(256, device="cuda")
    st = AdamW.init_state([w])
    make = lambda **kw: AdamW([w], **{**dict(weight_dtype="f32", grad_dtype="f32", **st), **kw})
    opt = make()
    for bad in (dict(m=[st["m"][0][:128]]), dict(m_scales=[st["m_scales"][0][:1]]), dict(m_scales=None),
                dict(weight_dtype="bf16"), dict(compute=[w]), dict(v=[])):
        with pytest.raises(ValueError):
            make(**bad)
    for bad in (dict(beta1=1.0), dict(eps=0.0), dict(weight_decay=-1.0)):
        with pytest.raises(RuntimeError):
            make(**bad)
    g = torch.zeros(256, device="cuda")
    for bad in ([g[:255]], [g.bfloat16()], [g, g], [g.cpu()], [torch.zeros(512, device="cuda")[::2]]):
        with pytest.raises(ValueError):
            opt.step(bad, 1, 1e-3)
    with pytest.raises(ValueError):
        opt.step([g], 1, 1e-3, grad_scale=torch.ones(1, device="cuda", dtype=torch.float64))
    for t, lr in ((0, 1e-3), (1, -1.0), (1, math.nan)):
        with pytest.raises(RuntimeError):
            opt.step([g], t, lr)
    norm = GradNorm([256], "f32")
    with pytest.raises(RuntimeError):
        norm([g], 0.0)
    with pytest.raises(ValueError):
        norm([g], out=torch.zeros(1, device="cuda"))


def test_refused_lists():
    """What a list's creation refuses, whatever tensor of it is at fault."""
    ws = [torch.zeros(k, device="cuda") for k in (5, 0, 300)]
    zeros = lambda: [torch.zeros_like(w) for w in ws]
    args = dict(weight_dtype="f32", grad_dtype="f32", state_dtype="f32")
    AdamW(ws, zeros(), zeros(), compute=[None, None, torch.zeros(300, device="cuda", dtype=torch.bfloat16)], **args)
    low = AdamW.init_state(ws)
    for m, kw in ((zeros()[:2], {}), ([*zeros()[:2], None], {}), ([*zeros()[:2], torch.zeros(300)], {}),
                  ([*zeros()[:2], torch.zeros(600, device="cuda")[::2]], {}), ([*zeros()[:2], zeros()[2].bfloat16()], {}),
                  (zeros(), dict(m_scales=low["m_scales"])), (zeros(), dict(compute=[None] * 2)),
                  (zeros(), dict(compute=[None, None, torch.zeros(299, device="cuda", dtype=torch.bfloat16)]))):
        with pytest.raises(ValueError):
            AdamW(ws, m, zeros(), **args, **kw)
    with pytest.raises(ValueError):
        AdamW(ws, **{**low, "v_scales": low["v_scales"][:2]}, weight_dtype="f32", grad_dtype="f32")


@pytest.fixture(scope="module")
def probe(tmp_path_factory):
    from paper_2607_10611_gb300 import builder as B
    out = tmp_path_factory.mktemp("root") / "libroot_probe.so"
    subprocess.run([B.nvcc(), *B.NVCC_FLAGS, "-shared", str(Path(__file__).parent / "cuda" / "root_probe.cu"), "-o", str(out)],
                   check=True)
    lib = ctypes.CDLL(str(out))
    U, P = ctypes.c_uint32, ctypes.c_void_p
    lib.root_probe.argtypes = lib.reciprocal_probe.argtypes = [U, U, P]
    lib.quotient_probe.argtypes = [P, P, ctypes.c_int64, P]
    return lib


def _bits(x):
    return int(np.float32(x).view(np.uint32))


def test_square_root_is_the_correctly_rounded_one_everywhere(probe):
    """Every binary32 value from 0 up to 2^32, where the step turns to the library's square root."""
    wrong = torch.zeros(1, dtype=torch.int64, device="cuda")
    assert probe.root_probe(0, _bits(2.0 ** 32), wrong.data_ptr()) == 0
    assert int(wrong) == 0, int(wrong)


def test_reciprocal_is_the_correctly_rounded_one_everywhere(probe):
    """Every binary32 value in [2^-100, 2^100]."""
    wrong = torch.zeros(1, dtype=torch.int64, device="cuda")
    assert probe.reciprocal_probe(_bits(2.0 ** -100), _bits(2.0 ** 100) - _bits(2.0 ** -100) + 1, wrong.data_ptr()) == 0
    assert int(wrong) == 0, int(wrong)


def test_quotient_is_the_correctly_rounded_one(probe):
    """Random operands over the range, and mantissas at either end, where quotients come closest to ties."""
    g = torch.Generator(device="cuda").manual_seed(0)
    n = 1 << 26
    for near in (False, True):
        ints = lambda lo, hi: torch.randint(lo, hi, (n,), device="cuda", generator=g, dtype=torch.int32)
        mantissa = (lambda: torch.where(ints(0, 2) == 1, ints(0, 64), (1 << 23) - 1 - ints(0, 64))) if near else \
            (lambda: ints(0, 1 << 23))
        d = ((ints(-60, 60) + 127) << 23 | mantissa()).view(torch.float32)
        a = ((ints(-60, 60) + 127) << 23 | mantissa()).view(torch.float32)
        wrong = torch.zeros(1, dtype=torch.int64, device="cuda")
        assert probe.quotient_probe(a.data_ptr(), d.data_ptr(), n, wrong.data_ptr()) == 0
        assert int(wrong) == 0, int(wrong)


@pytest.fixture(scope="module")
def rounding_probe(tmp_path_factory):
    from paper_2607_10611_gb300 import builder as B
    out = tmp_path_factory.mktemp("rounding") / "librounding_probe.so"
    subprocess.run([B.nvcc(), *B.NVCC_FLAGS, "-shared", str(Path(__file__).parent / "cuda" / "rounding_probe.cu"), "-o", str(out)],
                   check=True)
    lib = ctypes.CDLL(str(out))
    lib.codes_probe.argtypes = lib.pairs_probe.argtypes = [ctypes.c_void_p]
    return lib


@pytest.mark.parametrize("which", ["codes", "pairs"])
def test_stochastic_conversions_are_the_definition_everywhere(rounding_probe, which):
    """Codes for every value up to 448 and pairs for every finite one."""
    wrong = torch.zeros(1, dtype=torch.int64, device="cuda")
    assert getattr(rounding_probe, which + "_probe")(wrong.data_ptr()) == 0
    assert int(wrong) == 0, int(wrong)
