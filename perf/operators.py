"""Timed cases of the 8-bit training operators, through the package's public entry points.

Five operators, as a training or serving program calls them:

* "norm": the global norm of a list of gradients and the multiplier that clips them (adamw.GradNorm);
* "adamw": one AdamW step over a list of tensors with moments in binary32 or in 8 bits (adamw.AdamW);
* "quant": a matrix into E4M3 with a power-of-two scale per block of 128, as it lies and/or transposed (fp8.quantize);
* "matmul": the product of two such matrices (fp8.matmul);
* "linear": a linear layer in that format, forward and backward (fp8.linear).

Shapes are those of the repository's workloads (GPT-2 small, LLaMA-style decoders of 1.5B and 7B parameters) and generic
ones of the same kind.  Every rounding to 8 bits is defined bit for bit, in both forms below.
"""
import math
import random

import numpy as np
import torch

own = False

FIRST_STEP = 1000
LR, BETA1, BETA2, EPS, DECAY, MAX_NORM = 1e-3, 0.9, 0.999, 1e-8, 0.1, 1.0
BLOCK = 128
E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}


# ---------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------
def _gpt2(layers, d, vocab, ctx, group):
    vectors, matrices = [], [vocab * d, ctx * d]
    for _ in range(layers):
        vectors += [d, d, 3 * d, d, d, d, 4 * d, d]
        matrices += [3 * d * d, d * d, 4 * d * d, 4 * d * d]
    vectors += [d, d]
    return vectors if group == "vectors" else matrices if group == "matrices" else vectors + matrices


def _llama(layers, d, ffn, vocab):
    return [vocab * d] * (2 if vocab else 0) + ([d * d] * 4 + [d * ffn] * 3 + [d] * 2) * layers + [d]


def _ragged(tensors, max_log2, list_seed):
    r = random.Random(list_seed)
    return [max(1, round(math.exp(r.random() * max_log2 * math.log(2.0)))) for _ in range(tensors)]


def sizes(case):
    if case["list"] == "gpt2":
        return _gpt2(case["layers"], case["d"], case["vocab"], case["ctx"], case["group"])
    if case["list"] == "llama":
        return _llama(case["layers"], case["d"], case["ffn"], case["vocab"])
    return _ragged(case["tensors"], case["max_log2"], case["list_seed"])


def listed():
    gpt2 = {"list": "gpt2", "layers": 12, "d": 768, "vocab": 50257, "ctx": 1024}
    return [
        # Norms and biases of GPT-2 small, a group of their own without decay: the smallest step, all latency.
        dict(gpt2, name="adamw_vectors", op="adamw", group="vectors", weights="bf16", compute=False, grads="bf16",
             state="f32", rounding="nearest", state_rounding="nearest", clip=False, decay=0.0),
        # The whole of GPT-2 small in the usual mixed precision: binary32 weights and moments, BF16 gradients that the
        # multiplier clips, the BF16 copy for the next forward pass from the same step.
        dict(gpt2, name="adamw_gpt2_f32", op="adamw", group="all", weights="f32", compute=True, grads="bf16",
             state="f32", rounding="nearest", state_rounding="nearest", clip=True, decay=DECAY),
        # A 7B-width shard with 8-bit moments and BF16 weights, all rounded stochastically: the largest step.
        dict(name="adamw_llama_e4m3", op="adamw", list="llama", layers=2, d=4096, ffn=11008, vocab=32000,
             weights="bf16", compute=False, grads="bf16", state="e4m3", rounding="stochastic",
             state_rounding="stochastic", clip=True, decay=DECAY),
        # Clipping for the ragged list: 4000 tensors of 1 to 2^18 elements.
        dict(name="norm_ragged", op="norm", list="ragged", tensors=4000, max_log2=18, list_seed=1, grads="bf16"),
        # Clipping for a 7B-width shard.
        dict(name="norm_llama", op="norm", list="llama", layers=2, d=4096, ffn=11008, vocab=0, grads="bf16"),
        # Activations on their way into a layer: rows for the forward product, the transpose for the weight gradient.
        dict(name="quant_activations", op="quant", rows=8192, cols=4096, dtype="bf16", square=False, transposed=True),
        # GPT-2's embedding as a weight, in squares, in binary32 (rows are no multiple of 128).
        dict(name="quant_weight", op="quant", rows=50257, cols=768, dtype="f32", square=True, transposed=True),
        # The forward product of a 7B-width layer over 8192 tokens: the largest product.
        dict(name="matmul_forward", op="matmul", m=8192, n=11008, k=4096, out="bf16", accumulate=False),
        # A weight gradient of the 1.5B width over a ragged number of tokens, added to what earlier micro-batches left.
        dict(name="matmul_gradient", op="matmul", m=2048, n=5632, k=8119, out="f32", accumulate=True),
        # GPT-2's fused q, k, v projection over a ragged batch, forward and backward: many small calls.
        dict(name="linear_gpt2", op="linear", tokens=1023, k=768, n=2304, train=True),
        # A 1.5B-width projection over 8192 tokens, forward and backward.
        dict(name="linear_llama", op="linear", tokens=8192, k=2048, n=5632, train=True),
        # One token through a 7B-width layer in serving: the weight, held in 8 bits, is read once; nothing else counts.
        dict(name="linear_token", op="linear", tokens=1, k=4096, n=11008, train=False),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    def width(lo, hi):  # of a layer: a multiple of 64 as a rule, an odd size now and then
        n = log_int(lo, hi)
        return n if rng.random() < 0.25 else max(64, 64 * round(n / 64))

    op = rng.choice(["adamw", "adamw", "norm", "quant", "matmul", "matmul", "linear"])
    case = {"op": op}
    if op in ("adamw", "norm"):
        case["list"] = rng.choice(["gpt2", "llama", "ragged"])
        if case["list"] == "gpt2":
            case.update(layers=rng.randint(2, 24), d=64 * rng.randint(2, 18), vocab=log_int(1000, 50257),
                        ctx=log_int(128, 2048), group=rng.choice(["all", "all", "matrices", "vectors"]))
        elif case["list"] == "llama":
            d = 128 * rng.randint(1, 16)
            case.update(layers=rng.randint(1, 6), d=d, ffn=8 * round(d * rng.uniform(2.5, 4.0) / 8),
                        vocab=log_int(1000, 32000))
        else:
            case.update(tensors=log_int(1, 4000), max_log2=rng.randint(10, 18), list_seed=rng.randrange(1 << 20))
        case["grads"] = rng.choice(["bf16", "bf16", "f32"])
        if op == "adamw":
            case["weights"] = rng.choice(["bf16", "f32"])
            case["compute"] = case["weights"] == "f32" and rng.random() < 0.6
            case["state"] = rng.choice(["f32", "e4m3", "e4m3"])
            case["rounding"] = rng.choice(["nearest", "stochastic"])
            case["state_rounding"] = rng.choice(["nearest", "stochastic", "stochastic"]) if case["state"] == "e4m3" else "nearest"
            case["clip"] = rng.random() < 0.5
            case["decay"] = rng.choice([0.0, DECAY])
    elif op == "quant":
        case.update(rows=log_int(1, 16384), cols=width(64, 8192), dtype=rng.choice(["bf16", "bf16", "f32"]),
                    square=rng.random() < 0.4, transposed=rng.random() < 0.6)
    elif op == "matmul":
        case.update(m=log_int(1, 8192), n=width(64, 11008), k=width(64, 4096), out=rng.choice(["bf16", "bf16", "f32"]))
        case["accumulate"] = case["out"] == "f32" and rng.random() < 0.6
    else:
        case["train"] = rng.random() < 0.6
        case.update(tokens=log_int(1, 8192 if case["train"] else 256), k=width(64, 2048), n=width(64, 5632))
    return case


# ---------------------------------------------------------------------------
# The definitions that both forms share with their users: blocks, scales, random lanes (32-bit arithmetic)
# ---------------------------------------------------------------------------
def _pow2(k):
    """2^k as binary32, for whole k in [-126, 127]."""
    return ((k + 127) << 23).to(torch.int32).view(torch.float32)


def _exponent(a):
    """The smallest k with a <= 448 * 2^k, at least -127; 0 where a is 0."""
    frac, e = torch.frexp(a)
    k = e.to(torch.int32) - 9 + (frac > 0.875).to(torch.int32)
    return torch.where(a > 0, k, torch.zeros_like(k)).clamp(-127, 127)


def _finite_max(x, dim):
    return torch.where(torch.isfinite(x), x.abs(), torch.zeros_like(x)).amax(dim)


def _philox(c, seed):
    """Philox4x32-10 of the counters c (four int64 tensors or numbers) under the key `seed`: four int64 tensors of 32 bits."""
    m = 0xFFFFFFFF
    x0, x1, x2, x3 = c
    k0, k1 = seed & m, seed >> 32 & m
    for _ in range(10):
        p, q = x0 * 0xD2511F53, x2 * 0xCD9E8D57
        x0, x1, x2, x3 = (q >> 32 & m) ^ x1 ^ k0, q & m, (p >> 32 & m) ^ x3 ^ k1, p & m
        k0, k1 = (k0 + 0x9E3779B9) & m, (k1 + 0xBB67AE85) & m
    return x0, x1, x2, x3


def _weight_lanes(n, t, seed):
    """The 16 random bits of elements 0 .. n - 1 (n a multiple of 8): lane i mod 8 of block i div 8."""
    b = torch.arange(n // 8, dtype=torch.int64, device="cuda")
    z = torch.zeros_like(b)
    x = _philox((b, z, z + t, z), seed)
    return torch.stack([y for w in x for y in (w & 0xFFFF, w >> 16)], 1).reshape(-1)


def _state_lanes(n, t, seed):
    """The 32 random bits of elements 0 .. n - 1 (n a multiple of 4) for their moments: word i mod 4 of block i div 4 of
    the counters whose second word has its highest bit set."""
    b = torch.arange(n // 4, dtype=torch.int64, device="cuda")
    z = torch.zeros_like(b)
    return torch.stack(_philox((b, z + 0x80000000, z + t, z), seed), 1).reshape(-1)


def _to_e4m3(y, lanes=None):
    """Values, scaled already, as E4M3: nearest (ties to even), or stochastic by 16-bit lanes; saturating at 448."""
    if lanes is not None:
        a = y.abs()
        off = torch.where(a < 2.0 ** -6, 2.0 ** -6, 0.0).to(torch.float32)
        bits = (a + off).view(torch.int32)
        r = ((bits + (lanes.to(torch.int32) << 4)) & ~0xFFFFF).view(torch.float32) - off
        y = torch.where(a <= 448.0, torch.copysign(r, y), y)
    return y.clamp(-448.0, 448.0).to(E4M3)


def _to_e8m0(k):
    return (k + 127).to(torch.uint8).view(E8M0)


def _round_up(n, m):
    return -(-n // m) * m


def _tiled(k):
    """Exponents [rows, blocks] in the order they are stored in: tiles of 128 rows and 4 blocks, each [32][4][4] with row
    32 j + i's four blocks at [i][j]; 0 in the padding."""
    rows, blocks = k.shape
    k = torch.nn.functional.pad(k, (0, -blocks % 4, 0, -rows % BLOCK))
    return k.view(-1, 4, 32, k.shape[1] // 4, 4).permute(0, 3, 2, 1, 4).contiguous()


def _rows_exponents(scales, rows, blocks):
    """And back, as exponents [rows, blocks]."""
    k = scales.view(torch.uint8).to(torch.int32) - 127
    return k.permute(0, 3, 2, 1, 4).reshape(k.shape[0] * BLOCK, -1)[:rows, :blocks]


def _quantize(x, square):
    """Codes [rows, cols] (rows of a multiple of 16 bytes) and stored scales of the matrix x (binary32)."""
    rows, cols = x.shape
    p = torch.nn.functional.pad(x, (0, -cols % BLOCK, 0, -rows % BLOCK if square else 0))
    if square:
        p = p.view(p.shape[0] // BLOCK, BLOCK, -1, BLOCK)
        k = _exponent(_finite_max(p, (1, 3)))
        scaled = p * _pow2(-k)[:, None, :, None]
        k = k.repeat_interleave(BLOCK, 0)[:rows]
    else:
        p = p.view(rows, -1, BLOCK)
        k = _exponent(_finite_max(p, 2))
        scaled = p * _pow2(-k)[:, :, None]
    store = torch.zeros(rows, _round_up(cols, 16), dtype=E4M3, device=x.device)
    codes = store[:, :cols]
    codes.copy_(_to_e4m3(scaled.view(-1, p.shape[-2] * BLOCK)[:rows, :cols]))
    return codes, _to_e8m0(_tiled(k))


def _values(codes, scales):
    """What a quantised matrix stands for, in binary32."""
    rows, cols = codes.shape
    k = _rows_exponents(scales, rows, -(-cols // BLOCK))
    s = torch.where(k == -127, 2.0 ** -127, _pow2(k.clamp(min=-126)))
    return codes.float() * s.repeat_interleave(BLOCK, 1)[:, :cols]


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _matrix(rows, cols, gen, spread=0.0):
    """Normal values; with `spread`, columns differ in their scale, as activations' channels do."""
    x = torch.randn(rows, cols, generator=gen, device="cuda")
    if spread:
        x *= torch.exp(spread * torch.randn(cols, generator=gen, device="cuda"))
    return x


def _views(buf, ns):
    views, o = [], 0
    for n in ns:
        views.append(buf[o:o + n])
        o += _round_up(n, BLOCK)
    return views


def _prepare_list(case, seed):
    """Mid-training values in flat buffers, as a program that shards or reduces its parameters keeps them; every tensor
    starts at a multiple of 128 elements, and the padding is zero."""
    gen, host, ns = _generator(seed), random.Random(seed), sizes(case)
    total = sum(_round_up(n, BLOCK) for n in ns)
    lengths = torch.tensor([x for n in ns for x in (n, -n % BLOCK)], device="cuda")
    real = torch.tensor([1.0, 0.0], device="cuda").repeat(len(ns)).repeat_interleave(lengths)
    sd = [x for _ in ns for x in (math.exp(host.uniform(math.log(1e-5), math.log(1e-2))), 0.0)]
    sd = torch.tensor(sd, dtype=torch.float32, device="cuda").repeat_interleave(lengths)  # of each tensor's gradients

    def normal():
        return torch.randn(total, generator=gen, device="cuda")

    s = {"case": case, "ns": ns, "seed": seed, "t": FIRST_STEP, "g": (normal() * sd).to(TORCH[case["grads"]])}
    if case["op"] == "norm":
        if own:
            from paper_2607_10611_gb300.adamw import GradNorm
            s["norm"] = GradNorm(ns, case["grads"])
            s["grads"] = _views(s["g"], ns)
        return s
    s["w"] = (normal() * 0.02 * real).to(TORCH[case["weights"]])
    m = normal() * 0.3 * sd
    r = torch.empty(total, device="cuda").uniform_(0.5, 1.5, generator=gen) * sd
    del sd, real
    if case["state"] == "e4m3":  # the second moment is held by its root
        for name, x in (("m", m), ("v", r)):
            x = x.view(-1, BLOCK)
            k = _exponent(_finite_max(x, 1))
            q = _to_e4m3(x * _pow2(-k)[:, None])
            if name == "v":
                q = torch.where((x > 0) & (q.float() == 0), torch.full_like(x, 2.0 ** -9), q.float()).to(E4M3)
            s[name], s[name + "_scale"] = q.view(-1), _to_e8m0(k)
    else:
        s["m"], s["v"] = m, r.square_()
    if case["compute"]:
        s["compute"] = torch.zeros(total, dtype=torch.bfloat16, device="cuda")
    if case["clip"]:
        s["multiplier"] = torch.tensor([host.uniform(0.2, 1.0)], device="cuda")  # what the norm left, a tensor on the GPU
    if own:
        from paper_2607_10611_gb300.adamw import AdamW
        s["grads"] = _views(s["g"], ns)
        starts = dict(zip(("w", "m", "v"), ([*_views(s[name], ns)] for name in ("w", "m", "v"))))
        scales = {}
        if case["state"] == "e4m3":
            blocks = [-(-n // BLOCK) for n in ns]
            for name in ("m_scale", "v_scale"):
                scales[name + "s"] = list(torch.split(s[name], blocks))
        s["opt"] = AdamW(starts["w"], starts["m"], starts["v"], **scales, grad_dtype=case["grads"],
                         weight_dtype=case["weights"], state_dtype=case["state"], rounding=case["rounding"],
                         state_rounding=case["state_rounding"], seed=seed, beta1=BETA1, beta2=BETA2, eps=EPS,
                         weight_decay=case["decay"], compute=_views(s["compute"], ns) if case["compute"] else None)
    return s


def prepare(case, seed):
    if case["op"] in ("adamw", "norm"):
        return _prepare_list(case, seed)
    gen, s = _generator(seed), {"case": case}
    if case["op"] == "quant":
        if case["square"]:
            x = _matrix(case["rows"], case["cols"], gen) * 0.02
        else:
            x = _matrix(case["rows"], case["cols"], gen, 1.0)
        s["x"] = x.to(TORCH[case["dtype"]])
    elif case["op"] == "matmul":
        m, n, k = case["m"], case["n"], case["k"]
        if case["accumulate"]:  # a weight gradient: both operands are transposes, scaled along the tokens
            a, b = _matrix(m, k, gen) * 1e-3, _matrix(n, k, gen)
        else:
            a, b = _matrix(m, k, gen, 0.5), _matrix(n, k, gen) * 0.02
        s["a"] = _quantize(a.to(torch.bfloat16).float(), False)
        s["b"] = _quantize(b.to(torch.bfloat16).float(), not case["accumulate"])
        s["d"] = torch.zeros(m, n, dtype=TORCH[case["out"]], device="cuda")
        if case["accumulate"]:
            s["d"].normal_(generator=gen).mul_(1e-3 * math.sqrt(k))
    else:
        t, k, n = case["tokens"], case["k"], case["n"]
        s["x"] = _matrix(t, k, gen, 0.5).to(torch.bfloat16)
        s["w"] = (_matrix(n, k, gen) * 0.02).to(torch.bfloat16)
        s["dy"] = (_matrix(t, n, gen) * 1e-3).to(torch.bfloat16)
        if case["train"]:
            s["x"].requires_grad_()
            s["w"].requires_grad_()
        else:  # serving holds the weight in 8 bits
            s["b"] = _quantize(s["w"].float(), True)
    return s


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------
def _f32(x):
    return float(np.float32(x))


def _plain_adamw(s):
    case, t, seed = s["case"], s["t"], s["seed"]
    b1, b2 = _f32(BETA1), _f32(BETA2)
    omb1, omb2 = _f32(1.0 - b1), _f32(1.0 - b2)
    ka, c2 = _f32(_f32(LR) / (1.0 - b1 ** t)), _f32(1.0 / math.sqrt(1.0 - b2 ** t))
    kwd = _f32(_f32(LR) * _f32(case["decay"]))
    w, g = s["w"].float(), s["g"].float()
    if case["clip"]:
        g = g * s["multiplier"]
    low = case["state"] == "e4m3"
    if low:
        def old(name):
            k = s[name + "_scale"].view(torch.uint8).to(torch.int32) - 127
            p = torch.where(k == -127, 2.0 ** -127, _pow2(k.clamp(min=-126)))
            return (s[name].float().view(-1, BLOCK) * p[:, None]).view(-1)
        m, r = old("m"), old("v")
        v = r * r
    else:
        m, v = s["m"], s["v"]
    m = m * b1 + g * omb1
    v = v * b2 + (g * g) * omb2
    r = v.sqrt()
    u = (m * ka) / (r * c2 + _f32(EPS))
    w = (w - w * kwd if kwd else w) - u
    if low:
        lanes = None
        if case["state_rounding"] == "stochastic":
            lanes = _state_lanes(m.numel(), t, seed)
        for name, x in (("m", m), ("v", r)):
            x = x.view(-1, BLOCK)
            k = _exponent(_finite_max(x, 1))
            half = None if lanes is None else (lanes & 0xFFFF if name == "m" else lanes >> 16).view(-1, BLOCK)
            q = _to_e4m3(x * _pow2(-k)[:, None], half)
            if name == "v":
                q = torch.where((x > 0) & (q.float() == 0), torch.full_like(x, 2.0 ** -9), q.float()).to(E4M3)
            s[name].copy_(q.view(-1))
            s[name + "_scale"].copy_(_to_e8m0(k))
        del lanes
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)
    if case["weights"] == "bf16" and case["rounding"] == "stochastic":
        bits = w.view(torch.int32) + (0xFFFF - _weight_lanes(w.numel(), t, seed)).to(torch.int32)
        w = (bits & ~0xFFFF).view(torch.float32)
    s["w"].copy_(w)
    if case["compute"]:
        s["compute"].copy_(w)
    s["t"] = t + 1


def _plain_linear(s, a, b):
    """Forward product of the activations' values a and the weight's b."""
    return (a @ b.t()).to(torch.bfloat16)


def _adamw_outputs(s):
    return {k: s[k] for k in ("w", "m", "v", "m_scale", "v_scale", "compute") if k in s}


def _plain(s):
    case = s["case"]
    if case["op"] == "adamw":
        _plain_adamw(s)
        return _adamw_outputs(s)
    if case["op"] == "norm":
        n = s["g"].float().square().sum().sqrt()
        c = torch.where(torch.isfinite(n), (MAX_NORM / n).clamp(max=1.0), n - n)
        return torch.stack([n, c])
    if case["op"] == "quant":
        x = s["x"].float()
        return [*_quantize(x, case["square"]), *(_quantize(x.t(), case["square"]) if case["transposed"] else ())]
    if case["op"] == "matmul":
        p = _values(*s["a"]) @ _values(*s["b"]).t()
        if case["accumulate"]:
            s["d"] += p
        else:
            s["d"].copy_(p)
        return s["d"]
    x = s["x"].detach().float()
    if not case["train"]:
        return _plain_linear(s, _values(*_quantize(x, False)), _values(*s["b"]))
    w, dy = s["w"].detach().float(), s["dy"].float()
    wv = _values(*_quantize(w, True))
    y = _plain_linear(s, _values(*_quantize(x, False)), wv)
    dx = _values(*_quantize(dy, False)) @ wv
    dw = _values(*_quantize(dy.t(), False)) @ _values(*_quantize(x.t(), False)).t()
    return [y, dx.to(torch.bfloat16), dw.to(torch.bfloat16)]


def _framework(s):
    from paper_2607_10611_gb300 import fp8
    case = s["case"]
    if case["op"] == "adamw":
        s["opt"].step(s["grads"], s["t"], LR, grad_scale=s.get("multiplier"))
        s["t"] += 1
        return _adamw_outputs(s)
    if case["op"] == "norm":
        return s["norm"](s["grads"], MAX_NORM)
    if case["op"] == "quant":
        if case["transposed"]:
            q, qt = fp8.quantize(s["x"], square=case["square"], transposed=True)
            return [q.codes, q.scales, qt.codes, qt.scales]
        q = fp8.quantize(s["x"], square=case["square"])
        return [q.codes, q.scales]
    if case["op"] == "matmul":
        return fp8.matmul(fp8.E4M3Matrix(*s["a"]), fp8.E4M3Matrix(*s["b"]), out=s["d"], accumulate=case["accumulate"])
    if not case["train"]:
        return fp8.linear(s["x"], fp8.E4M3Matrix(*s["b"]))
    y = fp8.linear(s["x"], s["w"])
    dx, dw = torch.autograd.grad(y, (s["x"], s["w"]), s["dy"])
    return [y.detach(), dx, dw]


def run(state):
    return _framework(state) if own else _plain(state)


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------
def _stored(rows, cols):
    """Bytes of a quantised matrix: a byte per value, one per block of 128 in a row."""
    return rows * cols + rows * -(-cols // BLOCK)


def work(case):
    if case["op"] in ("adamw", "norm"):
        n = sum(sizes(case))
        if case["op"] == "norm":
            return {"bytes": n * SIZE[case["grads"]], "flops": 2 * n}
        state = 16 if case["state"] == "f32" else 4 * (1 + 1 / BLOCK)
        per = SIZE[case["grads"]] + 2 * SIZE[case["weights"]] + state + (2 if case["compute"] else 0)
        return {"bytes": int(n * per), "flops": 15 * n}
    if case["op"] == "quant":
        r, c = case["rows"], case["cols"]
        out = _stored(r, c) + (_stored(c, r) if case["transposed"] else 0)
        return {"bytes": r * c * SIZE[case["dtype"]] + out, "flops": 2 * r * c}
    if case["op"] == "matmul":
        m, n, k = case["m"], case["n"], case["k"]
        d = m * n * SIZE[case["out"]] * (2 if case["accumulate"] else 1)
        return {"bytes": _stored(m, k) + _stored(n, k) + d, "flops": 2 * m * n * k}
    t, k, n = case["tokens"], case["k"], case["n"]
    if not case["train"]:
        return {"bytes": 2 * t * k + _stored(n, k) + 2 * t * n, "flops": 2 * t * n * k}
    return {"bytes": 2 * (2 * t * k + 2 * n * k + 2 * t * n), "flops": 6 * t * n * k}


# ---------------------------------------------------------------------------
# The same in 64 bits, from the definitions
# ---------------------------------------------------------------------------
def _exact_exponent(a):
    """The smallest whole k >= -127 with a <= 448 * 2^k, found by trying; 0 for a = 0."""
    k = torch.floor(torch.log2(a.clamp(min=1e-300) / 448.0)) - 1
    for _ in range(3):
        k = torch.where(a > 448.0 * torch.exp2(k), k + 1, k)
    return torch.where(a > 0, k.clamp(-127, 127), torch.zeros_like(k))


def _exact_e4m3(y, lanes=None):
    """y on E4M3's grid: its spacing is 2^(e - 3) in [2^e, 2^(e + 1)), 2^-9 below 2^-6."""
    a = y.abs().clamp(max=448.0)
    e = torch.frexp(a.clamp(min=2.0 ** -6))[1] - 1
    step = torch.exp2((e - 3).double())
    n = a / step
    n = torch.round(n) if lanes is None else torch.floor(n + lanes.double() / 65536.0)  # round(): ties to even
    return torch.copysign((n * step).clamp(max=448.0), y)


def _exact_quantize(x, square):
    """(codes' values, exponents per row and block), both in 64 bits."""
    rows, cols = x.shape
    nb = -(-cols // BLOCK)
    p = torch.zeros(_round_up(rows, BLOCK), nb * BLOCK, dtype=torch.float64, device=x.device)
    p[:rows, :cols] = x
    a = p.abs().unflatten(1, (nb, BLOCK)).amax(2)
    if square:
        a = a.unflatten(0, (-1, BLOCK)).amax(1).repeat_interleave(BLOCK, 0)
    k = _exact_exponent(a)[:rows]
    q = _exact_e4m3(p[:rows] / torch.exp2(k).repeat_interleave(BLOCK, 1))
    return q[:, :cols], k


def _exact_values(x, square):
    q, k = _exact_quantize(x, square)
    return q * torch.exp2(k).repeat_interleave(BLOCK, 1)[:, :q.shape[1]]


def _exact_scales(k):
    """2^k in the stored order, by explicit indices; 1 in the padding."""
    rows, nb = k.shape
    out = torch.ones(-(-rows // BLOCK), -(-nb // 4), 32, 4, 4, dtype=torch.float64, device=k.device)
    r, b = torch.meshgrid(torch.arange(rows, device=k.device), torch.arange(nb, device=k.device), indexing="ij")
    out[r // 128, b // 4, r % 32, r % 128 // 32, b % 4] = torch.exp2(k)
    return out


def _exact_philox(c, seed):
    """Philox4x32-10 again, its products from 16-bit halves."""
    mask = 0xFFFFFFFF

    def product(x, m):
        lo, hi = x * (m & 0xFFFF), x * (m >> 16)
        return (hi + (lo >> 16)) >> 16, (((hi & 0xFFFF) << 16) + lo) & mask

    c, key = list(c), [seed & mask, seed >> 32]
    for r in range(10):
        h0, l0 = product(c[0], 0xD2511F53)
        h1, l1 = product(c[2], 0xCD9E8D57)
        keys = [(key[0] + r * 0x9E3779B9) & mask, (key[1] + r * 0xBB67AE85) & mask]
        c = [h1 ^ c[1] ^ keys[0], l1, h0 ^ c[3] ^ keys[1], l0]
    return c


def _exact_adamw(case, seed):
    s = prepare(case, seed)
    low, t = case["state"] == "e4m3", FIRST_STEP
    b1, b2, lr, wd, eps = (_f32(x) for x in (BETA1, BETA2, LR, case["decay"], EPS))
    g = s["g"].double()
    if case["clip"]:
        g = g * s["multiplier"].double()

    def old(name):
        return (s[name].double().view(-1, BLOCK) * s[name + "_scale"].double()[:, None]).view(-1)

    m, v = (old("m"), old("v").square_()) if low else (s["m"].double(), s["v"].double())
    m = m.mul_(b1).add_(g, alpha=1 - b1)
    v = v.mul_(b2).add_(g.square_(), alpha=1 - b2)
    del g
    r = v.sqrt()
    w = s["w"].double()
    w = w * (1 - lr * wd) - lr / (1 - b1 ** t) * m / (r / math.sqrt(1 - b2 ** t) + eps)
    got = {"w": w}
    if case["compute"]:
        got["compute"] = w
    if not low:
        return {**got, "m": m, "v": v}
    del v
    for name, x in (("m", m), ("v", r)):
        x = x.view(-1, BLOCK)
        k = _exact_exponent(x.abs().amax(1))
        lanes = None
        if case["state_rounding"] == "stochastic":
            i = torch.arange(x.numel() // 4, dtype=torch.int64, device="cuda")
            words = _exact_philox((i, 0 * i + (1 << 31), 0 * i + t, 0 * i), seed)
            lanes = torch.stack(words, 1).view(x.shape)
            del words, i
            lanes = lanes % 65536 if name == "m" else lanes // 65536
        q = _exact_e4m3(x / torch.exp2(k)[:, None], lanes)
        if name == "v":
            q = torch.where((x > 0) & (q == 0), torch.full_like(q, 2.0 ** -9), q)
        got[name], got[name + "_scale"] = q.view(-1), torch.exp2(k)
        del lanes
    return got


def exact(case, seed):
    if case["op"] == "adamw":
        return _exact_adamw(case, seed)
    s = prepare(case, seed)
    if case["op"] == "norm":
        n = math.sqrt(float(s["g"].double().square_().sum()))
        return torch.tensor([n, min(1.0, MAX_NORM / n) if n else 1.0], dtype=torch.float64)
    if case["op"] == "quant":
        got, x = [], s["x"].double()
        for y in (x, x.t()) if case["transposed"] else (x,):
            q, k = _exact_quantize(y, case["square"])
            got += [q, _exact_scales(k)]
        return got
    if case["op"] == "matmul":
        def value(codes, scales):
            r = torch.arange(codes.shape[0], device="cuda")[:, None]
            b = torch.arange(codes.shape[1], device="cuda")[None, :] // BLOCK
            return codes.double() * scales.double()[r // 128, b // 4, r % 32, r % 128 // 32, b % 4]
        p = value(*s["a"]) @ value(*s["b"]).t()
        return s["d"].double() + p if case["accumulate"] else p
    x, w, dy = (s[k].detach().double() for k in ("x", "w", "dy"))
    wv = _exact_values(w, True)
    y = _exact_values(x, False) @ wv.t()
    if not case["train"]:
        return y
    return [y, _exact_values(dy, False) @ wv, _exact_values(dy.t(), False) @ _exact_values(x.t(), False).t()]
