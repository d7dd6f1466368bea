"""The autograd functions and the example that runs them together."""
import os
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a CUDA device")]


def test_best_ratio_prefers_a_small_center_on_long_tails():
    from paper_2002_00104_b200 import training
    g = torch.Generator(device="cuda")
    g.manual_seed(0)
    flat = torch.rand(200, 512, generator=g, device="cuda") * 2 - 1
    tails = torch.randn(200, 512, generator=g, device="cuda") ** 3
    assert abs(training.best_ratio(flat) - 0.5) < 0.1          # uniform values: equal steps
    assert training.best_ratio(tails) < 0.3


def test_gradients_of_the_network_on_checkpoints():
    """Against PyTorch's own on the same network.  An 8-bit value is off by at most 1 / 126 of its
    group's range (a uniform error of 0.5 / 63 * 0.5 of it, rms 0.0023 m with m about 2.7 rms: 0.6 % of
    the rms); through the few operands of each gradient, and the 16-bit roundings of both networks,
    5 % of a gradient's norm leaves room for about six such errors added up."""
    import train_act8
    from paper_2002_00104_b200 import training
    width, blocks, tokens = 256, 2, 512
    x = torch.randn(tokens, width, device="cuda").bfloat16()
    t = torch.randn(tokens, width, device="cuda")
    settings = training.Checkpoints(group=64, ratio=0.5)

    def grads(forward):
        p = train_act8.parameters(width, blocks, 5)
        leaves = [v.requires_grad_() for group in p.values() for v in group]
        out = forward(p, x)
        return out, torch.autograd.grad((out.float() * t).sum(), leaves)

    out, want = grads(train_act8.forward_plain)
    out8, got = grads(lambda p, v: train_act8.forward_act8(p, v, settings))
    assert ((out8.float() - out.float()).norm() <= 0.02 * out.float().norm())
    for g, w in zip(got, want):
        assert g.dtype == w.dtype and g.shape == w.shape
        assert (g.float() - w.float()).norm() <= 0.05 * w.float().norm()


def test_the_example_trains_alike_in_less_memory():
    import train_act8
    _, (plain, kept16), (act8, kept8) = train_act8.run(steps=25, width=256, blocks=2, tokens=1024)
    assert act8[-1] < 0.7 * act8[0] and abs(act8[-1] - plain[-1]) < 0.1 * plain[-1]
    assert kept8 < 0.6 * kept16
