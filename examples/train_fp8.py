"""Trains a small two-layer network in 8 bits with the package's operators, as they are used together:

* the linear layers' products run on E4M3 matrices with a scale per block of 128 (fp8.linear), their weights' gradients
  are added up in binary32 over micro-batches;
* the gradients' global norm gives a multiplier on the GPU (GradNorm), which the step applies (nothing waits for it);
* AdamW holds binary32 weights, moments in 8 bits, and writes the BF16 weights that the next forward pass takes;
* the trained layers then serve single tokens from weights quantised once.

    python examples/train_fp8.py [--steps 200]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2607_10611_gb300 import AdamW, GradNorm, fp8  # noqa: E402


def train(steps=200, tokens=512, width=256, hidden=768, micro_batches=2, lr=2e-3, max_norm=1.0, seed=0):
    """Fits a random smooth function; returns (losses, the trained BF16 weights, a batch and its targets)."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    randn = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")
    shapes = [(hidden, width), (width, hidden)]
    master = [randn(n, k) * k ** -0.5 for n, k in shapes]
    weights = [w.to(torch.bfloat16).requires_grad_() for w in master]  # what the layers see
    grads = [torch.zeros_like(w) for w in master]
    optimizer = AdamW(master, **AdamW.init_state(master, "e4m3"), weight_dtype="f32", grad_dtype="f32",
                      compute=[w.detach() for w in weights], weight_decay=0.01, seed=seed)
    norm = GradNorm([g.numel() for g in grads], "f32")
    truth = randn(width, width) * width ** -0.5
    losses = []
    for t in range(1, steps + 1):
        torch._foreach_zero_(grads)
        total = torch.zeros((), device="cuda")
        for _ in range(micro_batches):
            x = randn(tokens, width).to(torch.bfloat16)
            target = torch.sin(x.float() @ truth)
            h = torch.nn.functional.gelu(fp8.linear(x, weights[0], grad_w=grads[0]))
            y = fp8.linear(h, weights[1], grad_w=grads[1])
            loss = (y.float() - target).square().mean() / micro_batches
            loss.backward()
            total += loss.detach()
        clip = norm(grads, max_norm)  # [norm, multiplier], on the GPU
        optimizer.step(grads, t, lr, grad_scale=clip[1:])
        losses.append(total)
    losses = torch.stack(losses).tolist()
    if optimizer.device_status() or fp8.device_status():
        raise RuntimeError("a kernel's bounded wait gave up")
    return losses, [w.detach() for w in weights], x, target


@torch.no_grad()
def serve(weights, x):
    """The network on single tokens, one after another, with weights quantised once."""
    held = [fp8.quantize(w, square=True) for w in weights]
    out = [fp8.linear(torch.nn.functional.gelu(fp8.linear(token[None], held[0])), held[1]) for token in x]
    return torch.cat(out)


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=200)
    args = ap.parse_args()
    losses, weights, x, target = train(steps=args.steps)
    for t in range(0, len(losses), max(1, len(losses) // 10)):
        print(f"step {t + 1:4d}  loss {losses[t]:.4f}")
    print(f"step {len(losses):4d}  loss {losses[-1]:.4f}")
    y = serve(weights, x[:16])
    print(f"16 tokens served one by one: loss {float((y.float() - target[:16]).square().mean()):.4f}")


if __name__ == "__main__":
    main()
