"""Timed cases of the operators around a decoder's matrices, through the package's public entry points.

Four operators, as a training or serving program calls them:

* "norm": layer normalisation over the last dimension, forward and backward, or forward alone (layer_norm);
* "orthogonal": a list of matrices, each by five Newton-Schulz steps nearly its polar factor (Orthogonalizer);
* "muon": one Muon step over a list of matrices: momentum, the same orthogonalisation, the weights' update (Muon);
* "fp4": tokens times a weight in NVFP4, as M+Adam's step leaves it (fp4.linear).

Shapes are those of the repository's workloads (GPT-2 small, LLaMA-style decoders of 1.5B and 7B parameters) and generic
ones of the same kind.
"""
import math
import random

import numpy as np
import torch

own = False

FIRST_STEP = 1000
EPS = 1e-5
LR, BETA, DECAY = 3e-4, 0.95, 0.1
COEFFICIENTS, STEPS = (3.4445, -4.7750, 2.0315), 5
GLOBAL_SCALE = 2.0 ** -10
GROUP = 16
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


# ---------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------
def shapes(case):
    """(rows, columns) of a case's matrices, as weights [out, in]."""
    if case["list"] == "one":
        return [(case["rows"], case["cols"])]
    if case["list"] == "gpt2":
        d = case["d"]
        return [(3 * d, d), (d, d), (4 * d, d), (d, 4 * d)] * case["layers"]
    if case["list"] == "llama":
        d, f = case["d"], case["ffn"]
        return ([(d, d)] * 4 + [(f, d)] * 2 + [(d, f)]) * case["layers"]
    r = random.Random(case["list_seed"])
    side = lambda: int(round(math.exp(r.uniform(math.log(case["smallest"]), math.log(case["largest"])))))
    return [(side(), side()) for _ in range(case["tensors"])]


def _products(rows, cols):
    """Multiply-adds of one matrix's steps: of X X^T and of A A, symmetric both, half; and B X."""
    m, n = min(rows, cols), max(rows, cols)
    return STEPS * (m * (m + 1) // 2 * (n + m) + m * m * n)


def listed():
    return [
        # One token of GPT-2 in serving: nothing but latency.
        dict(name="norm_token", op="norm", rows=1, cols=768, dtype="bf16", weights="bf16", bias=True, train=False),
        # A ragged batch of GPT-2's activations, forward and backward, binary32 weights beside BF16 activations.
        dict(name="norm_gpt2", op="norm", rows=1023, cols=768, dtype="bf16", weights="f32", bias=True, train=True),
        # Binary32 activations of an odd width, forward and backward.
        dict(name="norm_odd", op="norm", rows=4099, cols=1001, dtype="f32", weights="f32", bias=True, train=True),
        # A 7B-width decoder's activations, 16384 tokens, forward and backward: the largest.
        dict(name="norm_llama", op="norm", rows=16384, cols=4096, dtype="bf16", weights="bf16", bias=True, train=True),
        # Small matrices of odd sizes, wide and tall: latency.
        dict(name="orthogonal_ragged", op="orthogonal", list="ragged", tensors=6, smallest=100, largest=700, list_seed=3,
             dtype="bf16"),
        # A 7B-width down projection alone: the largest matrix.
        dict(name="orthogonal_llama", op="orthogonal", list="one", rows=4096, cols=11008, dtype="bf16"),
        # Half of GPT-2 small's hidden matrices, BF16 weights rounded stochastically, clipped gradients.
        dict(name="muon_gpt2", op="muon", list="gpt2", layers=6, d=768, weights="bf16", compute=False, grads="bf16",
             momentum="f32", rounding="stochastic", nesterov=True, clip=True, scale="rms"),
        # One layer of the 1.5B width in mixed precision: binary32 weights, their BF16 copy, BF16 momentum.
        dict(name="muon_llama", op="muon", list="llama", layers=1, d=2048, ffn=5632, weights="f32", compute=True,
             grads="f32", momentum="bf16", rounding="nearest", nesterov=True, clip=False, scale="rms"),
        # A small network's matrices of odd sizes, from a single row up.
        dict(name="muon_ragged", op="muon", list="ragged", tensors=12, smallest=1, largest=500, list_seed=8,
             weights="bf16", compute=False, grads="f32", momentum="f32", rounding="nearest", nesterov=False, clip=False, scale="spectral"),
        # One token through a 7B-width up projection in serving.
        dict(name="fp4_token", op="fp4", tokens=1, k=4096, n=11008, dtype="bf16"),
        # Four users' next tokens through GPT-2's fused q, k, v projection.
        dict(name="fp4_gpt2", op="fp4", tokens=4, k=768, n=2304, dtype="bf16"),
        # Seventeen tokens of a draft to be checked, through a 7B-width down projection.
        dict(name="fp4_draft", op="fp4", tokens=17, k=11008, n=4096, dtype="bf16"),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    def width(lo, hi):  # of a layer: a multiple of 64 as a rule, an odd size now and then
        n = log_int(lo, hi)
        return n if rng.random() < 0.25 else max(64, 64 * round(n / 64))

    op = rng.choice(["norm", "norm", "orthogonal", "muon", "muon", "fp4"])
    case = {"op": op}
    if op == "norm":
        case["cols"] = width(64, 8192)
        case["rows"] = min(log_int(1, 16384), 16000 * 4096 // case["cols"])
        case["dtype"] = rng.choice(["bf16", "bf16", "f32"])
        if case["dtype"] == "f32":
            case["rows"] = max(1, case["rows"] // 2)
        case["weights"] = rng.choice([case["dtype"], "f32"])
        case["bias"] = rng.random() < 0.7
        case["train"] = rng.random() < 0.7
    elif op == "fp4":
        case.update(tokens=log_int(1, 32), k=width(64, 11008), n=width(64, 11008), dtype=rng.choice(["bf16", "bf16", "f32"]))
        case["n"] = max(1, min(case["n"], 4096 * 11008 // case["k"], 17 * 4096 * 11008 // (case["tokens"] * case["k"])))
    else:
        case["list"] = rng.choice(["one", "gpt2", "llama", "ragged"])
        if case["list"] == "one":
            case.update(rows=width(16, 4096), cols=width(16, 4096))
        elif case["list"] == "gpt2":
            case.update(layers=rng.randint(1, 8), d=64 * rng.randint(1, 12))
            case["layers"] = min(case["layers"], 6) if case["d"] == 768 else case["layers"]
        elif case["list"] == "llama":
            d = 64 * rng.randint(2, 24)
            case.update(layers=1, d=d, ffn=8 * round(d * rng.uniform(2.5, 3.6) / 8))
        else:
            case.update(tensors=log_int(2, 40), smallest=log_int(1, 64), largest=log_int(64, 1000),
                        list_seed=rng.randrange(1 << 20))
        if op == "orthogonal":
            case["dtype"] = "bf16"
        else:
            case["weights"] = rng.choice(["bf16", "bf16", "f32"])
            case["compute"] = case["weights"] == "f32" and rng.random() < 0.6
            case["grads"] = rng.choice(["bf16", "f32"])
            case["momentum"] = rng.choice(["f32", "f32", "bf16"])
            case["rounding"] = rng.choice(["nearest", "stochastic"]) if case["weights"] == "bf16" else "nearest"
            case["nesterov"] = rng.random() < 0.7
            case["clip"] = rng.random() < 0.5
            case["scale"] = rng.choice(["rms", "rms", "spectral"]) if case["weights"] == "bf16" else "rms"
    return case


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
def _gradient(rows, cols, gen, sd):
    """A few strong directions and noise around them, as a linear layer's gradient over a batch has."""
    k = max(1, min(rows, cols) // 16)
    u = torch.randn(rows, k, generator=gen, device="cuda")
    v = torch.randn(k, cols, generator=gen, device="cuda")
    u *= torch.linspace(1.0, 0.1, k, device="cuda") / math.sqrt(k)
    return (u @ v + 0.3 * torch.randn(rows, cols, generator=gen, device="cuda")) * sd


def _prepare_list(case, seed):
    gen, host = torch.Generator(device="cuda").manual_seed(seed), random.Random(seed)
    sides = shapes(case)
    s = {"case": case, "shapes": sides, "seed": seed, "t": FIRST_STEP}
    sds = [math.exp(host.uniform(math.log(1e-5), math.log(1e-2))) for _ in sides]
    if case["op"] == "orthogonal":
        s["x"] = [_gradient(r, c, gen, sd).to(TORCH[case["dtype"]]) for (r, c), sd in zip(sides, sds)]
        if own:
            from paper_2607_10611_gb300 import Orthogonalizer
            s["orthogonalize"] = Orthogonalizer(sides, case["dtype"])
        return s
    s["g"] = [_gradient(r, c, gen, sd).to(TORCH[case["grads"]]) for (r, c), sd in zip(sides, sds)]
    s["m"] = [(0.3 * _gradient(r, c, gen, sd)).to(TORCH[case["momentum"]]) for (r, c), sd in zip(sides, sds)]
    s["w"] = [(0.02 * torch.randn(r, c, generator=gen, device="cuda")).to(TORCH[case["weights"]]) for r, c in sides]
    if case["compute"]:
        s["compute"] = [torch.zeros(r, c, dtype=torch.bfloat16, device="cuda") for r, c in sides]
    if case["clip"]:
        s["multiplier"] = torch.tensor([host.uniform(0.2, 1.0)], device="cuda")  # what the norm left, a tensor on the GPU
    if own:
        from paper_2607_10611_gb300 import Muon
        s["muon"] = Muon(s["w"], s["m"], weight_dtype=case["weights"], grad_dtype=case["grads"],
                         momentum_dtype=case["momentum"], rounding=case["rounding"], seed=seed, momentum=BETA,
                         nesterov=case["nesterov"], weight_decay=DECAY, scale=case["scale"], compute=s.get("compute"))
    return s


def prepare(case, seed):
    if case["op"] in ("orthogonal", "muon"):
        return _prepare_list(case, seed)
    gen, s = torch.Generator(device="cuda").manual_seed(seed), {"case": case}

    def normal(*size):
        return torch.randn(*size, generator=gen, device="cuda")

    if case["op"] == "norm":
        rows, cols = case["rows"], case["cols"]
        # channels differ in their scale and mean, rows too, as a residual stream's do
        x = normal(rows, cols) * torch.exp(0.5 * normal(cols)) + 0.5 * normal(cols)
        s["x"] = (x * torch.exp(0.5 * normal(rows, 1))).to(TORCH[case["dtype"]])
        s["w"] = (1.0 + 0.2 * normal(cols)).to(TORCH[case["weights"]])
        s["b"] = (0.1 * normal(cols)).to(TORCH[case["weights"]]) if case["bias"] else None
        if case["train"]:
            s["dy"] = (1e-3 * normal(rows, cols)).to(TORCH[case["dtype"]])
            for name in ("x", "w", "b"):
                if s[name] is not None:
                    s[name].requires_grad_()
        return s
    t, k, n = case["tokens"], case["k"], case["n"]
    s["x"] = (normal(t, k) * torch.exp(0.5 * normal(k))).to(TORCH[case["dtype"]])
    # the layout that M+Adam's step leaves: groups of 16 consecutive elements of the flat weight, two codes a byte
    w = torch.nn.functional.pad((0.02 * normal(n * k)), (0, -n * k % GROUP)).view(-1, GROUP)
    scale = (w.abs().amax(1) / (6.0 * GLOBAL_SCALE)).to(torch.float8_e4m3fn)
    y = w / (scale.float() * GLOBAL_SCALE)[:, None]
    middles = torch.tensor([(a + b) / 2 for a, b in zip(E2M1, E2M1[1:])], device="cuda")
    codes = (torch.bucketize(y.abs(), middles) | (y < 0).long() << 3).to(torch.uint8).view(-1, 2)
    s["codes"] = (codes[:, 0] | codes[:, 1] << 4)[:-(-n * k // 2)].contiguous()
    s["scales"] = scale.view(torch.uint8)
    if own:
        from paper_2607_10611_gb300 import fp4
        s["weight"] = fp4.NVFP4Matrix(s["codes"], s["scales"], GLOBAL_SCALE, (n, k))
    return s


# ---------------------------------------------------------------------------
# The plain forms
# ---------------------------------------------------------------------------
def _plain_norm(s):
    x, w = s["x"].detach().float(), s["w"].detach().float()
    mean = x.mean(1, keepdim=True)
    xc = x - mean
    rstd = 1.0 / (xc.square().mean(1, keepdim=True) + EPS).sqrt()
    n = xc * rstd
    y = n * w
    if s["b"] is not None:
        y = y + s["b"].detach().float()
    y = y.to(s["x"].dtype)
    if not s["case"]["train"]:
        return [y]
    dy = s["dy"].float()
    dn = dy * w
    dx = (dn - dn.mean(1, keepdim=True) - n * (dn * n).mean(1, keepdim=True)) * rstd
    got = [y, dx.to(s["x"].dtype), (dy * n).sum(0).to(s["w"].dtype)]
    return got + ([dy.sum(0).to(s["b"].dtype)] if s["b"] is not None else [])


def _plain_orthogonal(x):
    """Five steps X <- a X + (b A + c A A) X, A = X X^T, from X / |X|, on the side with fewer rows; binary32."""
    a, b, c = COEFFICIENTS
    tall = x.shape[0] > x.shape[1]
    x = x.t() if tall else x
    norm = x.double().square().sum().sqrt().float()
    x = torch.where(norm > 0, x / norm, x)
    for _ in range(STEPS):
        p = x @ x.t()
        x = a * x + (b * p + c * (p @ p)) @ x
    return x.t() if tall else x


def _philox(c, seed):
    """Philox4x32-10 of the counters c (four int64 tensors) under the key `seed`: four int64 tensors of 32 bits."""
    mask = 0xFFFFFFFF
    x0, x1, x2, x3 = c
    k0, k1 = seed & mask, seed >> 32 & mask
    for _ in range(10):
        p, q = x0 * 0xD2511F53, x2 * 0xCD9E8D57
        x0, x1, x2, x3 = (q >> 32 & mask) ^ x1 ^ k0, q & mask, (p >> 32 & mask) ^ x3 ^ k1, p & mask
        k0, k1 = (k0 + 0x9E3779B9) & mask, (k1 + 0xBB67AE85) & mask
    return x0, x1, x2, x3


def _lanes(first, n, t, seed):
    """The 16 random bits of elements first .. first + n - 1 (first a multiple of 8): lane i mod 8 of block i div 8."""
    block = first // 8 + torch.arange(-(-n // 8), dtype=torch.int64, device="cuda")
    z = torch.zeros_like(block)
    x = _philox((block & 0xFFFFFFFF, block >> 32, z + t, z), seed)
    return torch.stack([y for w in x for y in (w & 0xFFFF, w >> 16)], 1).reshape(-1)[:n]


def _lr_factor(case, rows, cols):
    return 0.2 * math.sqrt(max(rows, cols)) if case["scale"] == "rms" else math.sqrt(max(1.0, rows / cols))


def _f32(x):
    return float(np.float32(x))


def _plain_muon(s):
    case, t = s["case"], s["t"]
    beta = _f32(BETA)
    first = 0
    for i, (rows, cols) in enumerate(s["shapes"]):
        g = s["g"][i].float()
        if case["clip"]:
            g = g * s["multiplier"]
        m = s["m"][i].float() * beta + g * _f32(1.0 - beta)
        s["m"][i].copy_(m)
        o = _plain_orthogonal(m * beta + g * _f32(1.0 - beta) if case["nesterov"] else m)
        w = s["w"][i].float()
        w = w - w * _f32(_f32(LR) * _f32(DECAY)) - o * _f32(_f32(LR) * _lr_factor(case, rows, cols))
        if case["rounding"] == "stochastic":
            bits = w.view(torch.int32) + (0xFFFF - _lanes(first, rows * cols, t, s["seed"])).to(torch.int32).view(rows, cols)
            w = (bits & ~0xFFFF).view(torch.float32)
        s["w"][i].copy_(w)
        if case["compute"]:
            s["compute"][i].copy_(w)
        first += -(-rows * cols // 128) * 128
    s["t"] = t + 1


def _muon_outputs(s):
    return {k: s[k] for k in ("w", "m", "compute") if k in s}


def _plain_fp4(s):
    n, k = s["case"]["n"], s["case"]["k"]
    pairs = s["codes"].to(torch.int32)
    codes = torch.stack([pairs & 15, pairs >> 4], 1).view(-1)[:n * k]
    magnitudes = torch.tensor(E2M1, device="cuda")[(codes & 7).long()]
    values = torch.where(codes >= 8, -magnitudes, magnitudes)
    scales = s["scales"].view(torch.float8_e4m3fn).float() * GLOBAL_SCALE
    w = (values * scales.repeat_interleave(GROUP)[:n * k]).view(n, k)
    return (s["x"].float() @ w.t()).to(s["x"].dtype)


def _plain(s):
    op = s["case"]["op"]
    if op == "norm":
        return _plain_norm(s)
    if op == "orthogonal":
        return [_plain_orthogonal(x.float()).to(x.dtype) for x in s["x"]]
    if op == "fp4":
        return _plain_fp4(s)
    _plain_muon(s)
    return _muon_outputs(s)


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------
def _framework(s):
    case = s["case"]
    if case["op"] == "norm":
        from paper_2607_10611_gb300 import layer_norm
        y = layer_norm(s["x"], s["w"], s["b"], eps=EPS)
        if not case["train"]:
            return [y]
        return [y.detach(), *torch.autograd.grad(y, [v for v in (s["x"], s["w"], s["b"]) if v is not None], s["dy"])]
    if case["op"] == "orthogonal":
        return s["orthogonalize"](s["x"])
    if case["op"] == "fp4":
        from paper_2607_10611_gb300 import fp4
        return fp4.linear(s["x"], s["weight"])
    s["muon"].step(s["g"], s["t"], LR, grad_scale=s.get("multiplier"))
    s["t"] += 1
    return _muon_outputs(s)


def run(state):
    return _framework(state) if own else _plain(state)


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    if case["op"] == "norm":
        n, size = case["rows"] * case["cols"], SIZE[case["dtype"]]
        vectors = case["cols"] * SIZE[case["weights"]] * (2 if case["bias"] else 1)
        if not case["train"]:
            return {"bytes": 2 * n * size + vectors, "flops": 8 * n}
        return {"bytes": 4 * n * size + 2 * vectors, "flops": 24 * n}
    if case["op"] == "fp4":
        t, k, n = case["tokens"], case["k"], case["n"]
        return {"bytes": n * k // 2 + n * k // GROUP + t * (n + k) * SIZE[case["dtype"]], "flops": 2 * t * n * k}
    elements = sum(r * c for r, c in shapes(case))
    flops = sum(2 * _products(r, c) for r, c in shapes(case))
    if case["op"] == "orthogonal":
        return {"bytes": 2 * elements * SIZE[case["dtype"]], "flops": flops}
    per = SIZE[case["grads"]] + 2 * SIZE[case["momentum"]] + 2 * SIZE[case["weights"]] + (2 if case["compute"] else 0)
    return {"bytes": elements * per, "flops": flops}


# ---------------------------------------------------------------------------
# The same in 64 bits, from the definitions
# ---------------------------------------------------------------------------
def _exact_norm(s):
    x, w = s["x"].detach().double(), s["w"].detach().double()
    d = x.shape[1]
    mu = x.sum(1) / d
    var = (x * x).sum(1) / d - mu * mu
    sigma = torch.sqrt(var + EPS)
    z = (x - mu[:, None]) / sigma[:, None]
    y = torch.addcmul(s["b"].detach().double()[None], z, w) if s["b"] is not None else z * w
    if not s["case"]["train"]:
        return [y]
    dy = s["dy"].double()
    h = torch.einsum("rc,c->rc", dy, w)
    along, total = torch.einsum("rc,rc->r", h, z), h.sum(1)
    dx = (d * h - total[:, None] - along[:, None] * z) / (d * sigma[:, None])
    got = [y, dx, torch.einsum("rc,rc->c", dy, z)]
    return got + ([torch.einsum("rc->c", dy)] if s["b"] is not None else [])


def _exact_orthogonal(x):
    """By the Gram matrix of the shorter side: the steps' polynomials of it multiply up to one factor of X."""
    a, b, c = COEFFICIENTS
    left = x.shape[0] <= x.shape[1]
    norm = float(torch.linalg.vector_norm(x))
    x = x / norm if norm else x
    for _ in range(STEPS):
        gram = x @ x.mT if left else x.mT @ x
        factor = c * gram
        factor.diagonal().add_(b)
        factor = factor @ gram
        factor.diagonal().add_(a)
        x = factor @ x if left else x @ factor
    return x


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        return _exact_norm(s)
    if case["op"] == "orthogonal":
        return [_exact_orthogonal(x.double()) for x in s["x"]]
    if case["op"] == "fp4":
        n, k = case["n"], case["k"]
        at = torch.arange(n * k, device="cuda")
        code = (s["codes"][at // 2].long() >> 4 * (at % 2)) & 15
        e, f = code // 2 % 4, code % 2
        value = torch.where(e > 0, torch.exp2(e.double() - 1) * (1 + f / 2.0), f / 2.0) * (1 - 2 * (code // 8)).double()
        group = s["scales"].view(torch.float8_e4m3fn).double() * GLOBAL_SCALE
        return s["x"].double() @ (value * group[at // GROUP]).view(n, k).mT
    beta, lr, decay = _f32(BETA), _f32(LR), _f32(DECAY)
    got = {"w": [], "m": []}
    for i, (rows, cols) in enumerate(s["shapes"]):
        g = s["g"][i].double()
        if case["clip"]:
            g = g * s["multiplier"].double()
        m = beta * s["m"][i].double() + (1 - beta) * g
        got["m"].append(m)
        o = _exact_orthogonal(beta * m + (1 - beta) * g if case["nesterov"] else m)
        factor = 0.2 * max(rows, cols) ** 0.5 if case["scale"] == "rms" else max(1.0, rows / cols) ** 0.5
        got["w"].append((1 - lr * decay) * s["w"][i].double() - lr * factor * o)
    if case["compute"]:
        got["compute"] = got["w"]
    return got
