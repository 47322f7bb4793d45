"""Norm, layers, gradients' norm, Muon and AdamW together, as a training step uses them: the block's gradients against plain ones,
the step against its formulas in 64 bits, eager and captured; and the example that trains so."""
import importlib.util
from pathlib import Path

import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2607_10611_gb300 import AdamW, GradNorm, Muon, fp8, layer_norm  # noqa: E402

from test_gpu_muon import _polar  # noqa: E402


@pytest.fixture(scope="module")
def example():
    path = Path(__file__).resolve().parents[1] / "examples" / "train_fp8.py"
    spec = importlib.util.spec_from_file_location("train_fp8", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def _block(seed=0, tokens=200, width=256, hidden=384):
    g = torch.Generator(device="cuda").manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")
    x = randn(tokens, width).bfloat16()
    weights = [(randn(n, k) * k ** -0.5).bfloat16() for n, k in [(hidden, width), (width, hidden)]]
    vectors = [1 + 0.2 * randn(width), 0.1 * randn(width)]
    return x, weights, vectors, randn(tokens, width).bfloat16()


def test_a_blocks_gradients(example):
    """Against the same block in 64 bits: what 8-bit products and BF16 activations cost.  E4M3 rounds a value by at most 2^-4,
    uniformly and so by 2^-4 / sqrt(3) = 0.036 at most as a root mean square; a product of two such matrices is off by
    sqrt(2) 0.036 = 0.051 of its 2-norm, a gradient goes through up to five of them (forward 2, backward 3): 0.114."""
    x, weights, vectors, dy = _block()
    leaves = [t.clone().requires_grad_() for t in (x, *weights, *vectors)]
    y = example.forward(leaves[0], leaves[1:3], leaves[3:])
    got = torch.autograd.grad(y, leaves, dy)
    plain = [t.double().requires_grad_() for t in (x, *weights, *vectors)]
    n = torch.nn.functional.layer_norm(plain[0], (256,), plain[3], plain[4], 1e-5)
    z = plain[0] + torch.nn.functional.gelu(n @ plain[1].t()) @ plain[2].t()
    for a, b, leaf in zip(got, torch.autograd.grad(z, plain, dy.double()), leaves):
        assert a.dtype == leaf.dtype and a.shape == leaf.shape
        assert float((a.double() - b).norm() / b.norm()) <= 0.114


def _state(seed=0):
    x, weights, vectors, dy = _block(seed)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    grads = [1e-2 * torch.randn(t.shape, generator=g, device="cuda") for t in (*weights, *vectors)]
    master = [w.float() for w in weights]
    muon = Muon(master, **Muon.init_state(master), weight_dtype="f32", grad_dtype="f32", compute=weights, weight_decay=0.1)
    adamw = AdamW(vectors, **AdamW.init_state(vectors, "f32"), weight_dtype="f32", grad_dtype="f32", weight_decay=0.0)
    norm = GradNorm([t.numel() for t in grads], "f32")
    out = torch.empty(2, device="cuda")

    def step():
        norm(grads, 1.0, out=out)
        muon.step(grads[:2], 1, 1e-2, grad_scale=out[1:])
        adamw.step(grads[2:], 1, 1e-2, grad_scale=out[1:])
    return step, master, weights, vectors, grads, (muon, adamw, norm, out)


def test_a_step_of_all_of_them():
    step, master, weights, vectors, grads, keep = _state()
    before = [w.clone() for w in master]
    total = torch.stack([g.double().square().sum() for g in grads]).sum().sqrt()
    step()
    torch.cuda.synchronize()
    assert keep[0].device_status() == 0
    for old, new, w, g in zip(before, master, weights, grads):
        m = 0.05 * g.double() / total.clamp(min=1.0)
        u = 0.95 * m + 0.05 * g.double() / total.clamp(min=1.0)
        want = old.double() * (1 - 1e-3) - 1e-2 * 0.2 * max(old.shape) ** 0.5 * _polar(u)
        moved = (want - old.double()).norm()
        # (the update is off by what test_gpu_muon's matrices are; the sums and products around it round in binary32)
        assert float((new.double() - want).norm()) <= 3e-3 * float(moved) + 2 ** -23 * float(want.norm())
        assert torch.equal(w, new.bfloat16())


def test_captured_it_gives_the_same_bits():
    eager = _state()
    for _ in range(3):
        eager[0]()
    captured = _state()
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        captured[0]()
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    for a, b in zip((*eager[1], *eager[2], *eager[3]), (*captured[1], *captured[2], *captured[3])):
        assert torch.equal(a, b)


def test_the_example_runs(example):
    losses, weights, vectors, x, target = example.train_with_muon(steps=6)
    assert len(losses) == 6 and all(l == l and abs(l) < 1e3 for l in losses)
    assert example.train_with_muon(steps=3)[0] == losses[:3]
    with torch.no_grad():
        assert example.forward(x, weights, vectors).shape == target.shape
