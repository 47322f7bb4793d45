"""The 8-bit linear layer's place in torch's graph: what it refuses, what it computes when only a part of its gradients
is asked for, what saved-tensor hooks see of it, and on which streams its results are ready."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2607_10611_gb300 import fp8  # noqa: E402


@pytest.fixture(autouse=True)
def waits_held():
    yield
    if torch.cuda.is_available():
        assert fp8.device_status() == 0


def _layer(tokens=24, k=96, n=40, seed=0, dtype=torch.bfloat16):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(tokens, k, generator=g).to(dtype).cuda().requires_grad_()
    w = (0.05 * torch.randn(n, k, generator=g)).to(dtype).cuda().requires_grad_()
    return x, w, torch.randn(tokens, n, generator=g).to(dtype).cuda()


@pytest.mark.parametrize("which", ["x", "w", "held"])
def test_tangents_are_refused(which):
    """A result without a tangent stands for a derivative of zero in forward mode."""
    x, w, _ = _layer()
    x, w = x.detach(), w.detach()
    held = fp8.quantize(w, square=True)
    want = fp8.linear(x, w)
    with torch.autograd.forward_ad.dual_level():
        dual = torch.autograd.forward_ad.make_dual(w if which == "w" else x, torch.ones_like(w if which == "w" else x))
        call = {"x": lambda: fp8.linear(dual, w), "w": lambda: fp8.linear(x, dual), "held": lambda: fp8.linear(dual, held)}[which]
        with pytest.raises(RuntimeError, match="forward"):
            call()
        with torch.autograd.forward_ad._set_fwd_grad_enabled(False):  # tangents are of no matter here, to torch either
            assert torch.equal(call(), want)
        assert torch.equal(fp8.linear(x, w), want)


def test_only_the_gradients_that_are_asked_for():
    """With a buffer for w's gradient: asking for x's leaves the buffer alone, and a following pass adds once."""
    x, w, dy = _layer(130)
    once = torch.zeros(40, 96, device="cuda")
    fp8.linear(x, w, grad_w=once).backward(dy)
    total = torch.zeros(40, 96, device="cuda")
    y = fp8.linear(x, w, grad_w=total)
    dx, = torch.autograd.grad(y, x, dy, retain_graph=True)
    assert torch.equal(total, torch.zeros_like(total))
    x.grad = None
    torch.autograd.backward(y, dy, inputs=[x], retain_graph=True)
    assert torch.equal(total, torch.zeros_like(total)) and torch.equal(x.grad, dx)
    y.backward(dy)
    assert torch.equal(total, once) and torch.equal(x.grad, dx + dx)


def test_no_product_is_made_for_a_gradient_nobody_asks_for():
    """By the memory that a backward pass takes: dx is 32 MiB here, dw 32 KiB."""
    x, w, dy = _layer(16384, 1024, 16)
    for asked, other in ((w, x), (x, w)):
        y = fp8.linear(x, w)
        torch.cuda.synchronize()
        torch.cuda.reset_peak_memory_stats()
        before = torch.cuda.memory_allocated()
        got, = torch.autograd.grad(y, asked, dy)
        taken = torch.cuda.max_memory_allocated() - before
        if asked is w:
            assert taken < x.numel() * x.element_size()  # no dx
        assert got.shape == asked.shape
        both = torch.autograd.grad(fp8.linear(x, w), (asked, other), dy)
        assert torch.equal(got, both[0])


def test_a_buffer_for_the_gradient_of_a_weight_without_one_is_refused():
    x, w, dy = _layer()
    total = torch.zeros(40, 96, device="cuda")
    with pytest.raises(ValueError, match="grad_w"):
        fp8.linear(x, w.detach(), grad_w=total)
    with pytest.raises(ValueError, match="grad_w"):
        fp8.linear(x.detach(), w.detach(), grad_w=total)
    with torch.no_grad():  # nothing is differentiated here
        assert torch.equal(fp8.linear(x, w, grad_w=total), fp8.linear(x, w.detach()))
    assert torch.equal(total, torch.zeros_like(total))
