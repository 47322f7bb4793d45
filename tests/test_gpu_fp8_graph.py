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


def test_saved_tensor_hooks_see_what_the_backward_pass_takes():
    x, w, dy = _layer(512, 1000, 400)
    want = torch.autograd.grad(fp8.linear(x, w), (x, w), dy)
    packed = []

    def pack(t):
        packed.append(t.numel() * t.element_size())
        return t.cpu()

    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    with torch.autograd.graph.saved_tensors_hooks(pack, lambda t: t.cuda()):
        y = fp8.linear(x, w)
    held = torch.cuda.memory_allocated() - before - 512 * 400 * 2
    assert len(packed) == 2 and sum(packed) >= 512 * 1000 + 1000 * 400  # x's and w's transposes in 8 bits
    assert held < 4096  # nothing of them stays on the GPU
    for _ in range(2):
        got = torch.autograd.grad(y, (x, w), dy, retain_graph=True)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    with torch.autograd.graph.save_on_cpu():
        y = fp8.linear(x, w)
    assert all(torch.equal(a, b) for a, b in zip(torch.autograd.grad(y, (x, w), dy), want))
    with pytest.raises(RuntimeError, match="second time"):
        torch.autograd.grad(y, (x, w), dy)


def test_a_hook_that_gives_something_else_back_is_refused():
    x, w, dy = _layer()
    for other in (lambda t: t[:-1], lambda t: t.cpu(), lambda t: t.float(), lambda t: t.view(1, -1)):
        with torch.autograd.graph.saved_tensors_hooks(lambda t: t, other):
            y = fp8.linear(x, w)
        with pytest.raises(RuntimeError, match="hook"):
            torch.autograd.grad(y, (x, w), dy)


def test_a_recomputed_layer_saves_nothing_and_gives_the_same():
    x, w, dy = _layer(512, 1000, 400)
    want = torch.autograd.grad(torch.nn.functional.gelu(fp8.linear(x, w)), (x, w), dy)
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    y = torch.utils.checkpoint.checkpoint(lambda a: torch.nn.functional.gelu(fp8.linear(a, w)), x, use_reentrant=False)
    assert torch.cuda.memory_allocated() - before < 512 * 400 * 2 + 4096
    got = torch.autograd.grad(y, (x, w), dy)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_a_buffer_for_the_gradient_is_ready_where_the_backward_call_returns():
    """The layer runs on another stream, which is busy, and w's place in the graph was made on this one: what reads the
    buffer here next has to see the sum."""
    x, w, dy = _layer(512, 1000, 400)
    x = x.detach()
    once = torch.zeros(400, 1000, device="cuda")
    fp8.linear(x, w, grad_w=once).backward(dy)
    accumulator = w.expand_as(w).grad_fn.next_functions[0][0]
    total = torch.zeros(400, 1000, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y = fp8.linear(x, w, grad_w=total)
        assert y.grad_fn.next_functions[1][0] is accumulator
        torch.cuda._sleep(100_000_000)  # about 50 ms
    y.backward(dy)
    got = total.clone()
    torch.cuda.synchronize()
    assert torch.equal(got, once) and w.grad is None


@pytest.mark.parametrize("shape,n", [((2, 3, 0), 5), ((4, 0), 5), ((0,), 5), ((0, 3, 0), 5), ((2, 3, 16), 0), ((16,), 0)])
def test_widths_of_zero(shape, n):
    """As torch's own linear: a sum of nothing is zero, and so is its gradient."""
    x = torch.ones(shape, device="cuda", requires_grad=True)
    w = torch.ones(n, shape[-1], device="cuda", requires_grad=True)
    y = fp8.linear(x, w)
    assert y.shape == (*shape[:-1], n) and torch.equal(y, torch.zeros_like(y))
    dx, dw = torch.autograd.grad(y, (x, w), torch.ones_like(y))
    assert torch.equal(dx, torch.zeros_like(x)) and torch.equal(dw, torch.zeros_like(w))
    with torch.no_grad():
        assert torch.equal(fp8.linear(x, fp8.quantize(w, square=True)), torch.zeros_like(y))


@pytest.mark.parametrize("rows,cols", [(0, 5), (5, 0), (0, 0), (0, 600)])
def test_values_of_empty_matrices(rows, cols):
    q = fp8.quantize(torch.ones(rows, cols, device="cuda"))
    assert q.row_scales().shape == (rows, -(-cols // 128)) and q.dequantize().shape == (rows, cols)


@pytest.mark.parametrize("tokens,k,n", [(129, 512, 700), (300, 130, 257), (1500, 1000, 2600), (4096, 256, 1100)])
def test_prompts_through_a_held_weight(tokens, k, n):
    """More tokens than one tile of a, by single CTAs and by pairs: bit for bit what the weight itself gives."""
    x, w, _ = _layer(tokens, k, n, 5)
    with torch.no_grad():
        held = fp8.quantize(w, square=True)
        want = fp8.linear(x, w)
        assert torch.equal(fp8.linear(x, held), want)
        assert torch.equal(fp8.linear(x.view(1, tokens, k), held), want[None])
        assert torch.equal(fp8.linear(x[3:4], held), want[3:4])
