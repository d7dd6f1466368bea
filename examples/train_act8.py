"""Trains a small residual network twice, with activations kept in 16 bits by PyTorch and in 8-bit
checkpoints, and prints both loss curves and what either keeps between forward and backward.

    python examples/train_act8.py [--steps 60] [--width 1024] [--blocks 4] [--tokens 4096]

Synthetic data: a fixed random teacher; the student has to match its outputs.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2002_00104_b200 import training  # noqa: E402


def parameters(width, blocks, seed, device="cuda"):
    g = torch.Generator(device=device)
    g.manual_seed(seed)

    def normal(*shape, std):
        return (torch.randn(*shape, generator=g, device=device) * std).bfloat16()

    p = {"pre": [], "post": [], "gate": [], "up": [], "down": []}
    for _ in range(blocks):
        p["pre"].append(torch.ones(width, device=device).bfloat16())
        p["post"].append(torch.ones(width, device=device).bfloat16())
        p["gate"].append(torch.full((1, width), 0.5, device=device).bfloat16())
        p["up"].append(normal(2 * width, width, std=width ** -0.5))
        p["down"].append(normal(width, 2 * width, std=(2 * width) ** -0.5))
    p["pre"].append(torch.ones(width, device=device).bfloat16())
    return p


def norm(v, w, eps=1e-6):
    v = v.float()
    return v * torch.rsqrt(v.square().mean(1, keepdim=True) + eps) * w.float()


def forward_plain(p, x):
    """The network in PyTorch operations; autograd keeps 16- and 32-bit activations."""
    r, h = x, norm(x, p["pre"][0]).to(x.dtype)
    for i, up in enumerate(p["up"]):
        f = torch.nn.functional.silu(h @ up.t()) @ p["down"][i].t()
        r32 = r.float() + p["gate"][i].float() * norm(f, p["post"][i])
        r, h = r32.to(x.dtype), norm(r32, p["pre"][i + 1]).to(x.dtype)
    return h


def forward_act8(p, x, settings):
    """The same on 8-bit checkpoints."""
    r, h = training.block_norm(x, None, p["pre"][0], settings=settings)
    for i, up in enumerate(p["up"]):
        f = training.linear(training.silu(training.linear(h, up, settings), settings),
                            p["down"][i], settings)
        r, h = training.block_norm(r, f, p["pre"][i + 1], p["post"][i], p["gate"][i],
                                   settings=settings)
    return h


def train(forward, student, x, target, steps, lr=2e-2):
    """Loss after each step, and the bytes that the first forward pass left behind for backward."""
    leaves = [t.requires_grad_() for group in student.values() for t in group]
    losses, kept, out, loss, grads = [], 0, None, None, None
    for step in range(steps):
        del out, loss, grads                      # so that what is counted below is this step's alone
        before = torch.cuda.memory_allocated()
        out = forward(student, x)
        loss = (out.float() - target).square().mean()
        if step == 1:
            kept = torch.cuda.memory_allocated() - before
        grads = torch.autograd.grad(loss, leaves)
        with torch.no_grad():
            for t, g in zip(leaves, grads):
                # one learning rate for all, on gradients of one size
                t.sub_((lr * g.float() / (g.float().square().mean().sqrt() + 1e-12)
                        * t.float().square().mean().sqrt()).to(t.dtype))
        losses.append(float(loss.detach()))
    return losses, kept


def run(steps=60, width=1024, blocks=4, tokens=4096):
    teacher = parameters(width, blocks, 1)
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    x = torch.randn(tokens, width, generator=g, device="cuda").bfloat16()
    with torch.no_grad():
        target = forward_plain(teacher, x).float()
    settings = training.Checkpoints(group=128, ratio=training.best_ratio(x[:256]))
    plain = train(forward_plain, parameters(width, blocks, 2), x, target, steps)
    act8 = train(lambda p, v: forward_act8(p, v, settings), parameters(width, blocks, 2), x, target, steps)
    return settings, plain, act8


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, default in (("steps", 60), ("width", 1024), ("blocks", 4), ("tokens", 4096)):
        ap.add_argument("--" + name, type=int, default=default)
    a = ap.parse_args()
    settings, (plain, kept16), (act8, kept8) = run(a.steps, a.width, a.blocks, a.tokens)
    print("checkpoints: group %d, breakpoint at %.4f of the range" % (settings.group, settings.ratio))
    print("kept for backward: %.1f MB in 16 / 32 bits, %.1f MB in 8-bit checkpoints" % (kept16 / 1e6, kept8 / 1e6))
    for step in range(0, a.steps, max(1, a.steps // 10)):
        print("step %4d   loss %.5f   with 8-bit checkpoints %.5f" % (step, plain[step], act8[step]))
    print("last        loss %.5f   with 8-bit checkpoints %.5f" % (plain[-1], act8[-1]))
