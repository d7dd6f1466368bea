"""PyTorch autograd functions over the training calls: what they keep between the forward and the
backward pass is 8-bit checkpoints, one byte per activation and one range per group.

``ratio`` is the breakpoint of the checkpoints' quantizer as a part of a group's range; ``best_ratio``
finds it with the library's breakpoint search on a sample of the activations.

The functions are differentiable once: in their gradients the kept activations are constants, so a
second derivative would lack terms, and asking for one raises.
"""
from __future__ import annotations

import torch
from torch.autograd.function import once_differentiable

from . import pwlq


class Checkpoints:
    """Settings of the checkpoints of a model: group length, breakpoint ratio."""

    def __init__(self, group: int = 128, ratio: float = 0.5):
        self.group, self.ratio = group, ratio


def best_ratio(x: torch.Tensor, group: int = 128, candidates: int = 32, bits: int = 7) -> float:
    """The breakpoint ratio with the smallest total squared error on x [rows, cols], or on several
    matrices [matrices, rows, cols] together.  Every group is a row of the search with this many bits: 7
    for checkpoints, 3 for 4-bit weights.  The last values of a row that do not fill a group are left out;
    rows shorter than a group are one each.  Candidates are k / candidates, the last one (no tail) left
    out."""
    if x.dim() not in (2, 3):
        raise ValueError(f"x must be [rows, cols] or [matrices, rows, cols], it is {list(x.shape)}")
    if x.numel() == 0 or candidates < 2:
        raise ValueError(f"no candidates, or no values: x is {list(x.shape)}")
    group = min(group, x.shape[-1])
    cols = x.shape[-1] // group * group
    rows = x[..., :cols].float().reshape(-1, group).contiguous()
    ratios = torch.arange(1, candidates, device=x.device, dtype=torch.float32) / candidates
    sse = pwlq.search(rows, bits, ratios, want_sse=True)["sse"]
    return float(ratios[sse.double().sum(dim=0).argmin()])


# Checkpoints and weights are kept through autograd: released when backward has used them, refused a
# second time unless the graph is retained, seen by saved-tensor hooks (which may hand back other
# memory), and weights checked for changes in place.
def _keep(ctx, saved, *tensors):
    memory, ctx.layout = saved.detached()
    ctx.save_for_backward(memory, *tensors)


def _kept(ctx):
    memory, *tensors = ctx.saved_tensors
    return (ctx.layout.attached(memory), *tensors)


class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, settings):
        saved = pwlq.act8_encode(x, group=settings.group, ratio=settings.ratio)
        _keep(ctx, saved, weight)
        return x @ weight.t()

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        saved, weight = _kept(ctx)
        dx = dy @ weight if ctx.needs_input_grad[0] else None
        dw = pwlq.act8_weight_grad(dy.contiguous(), saved) if ctx.needs_input_grad[1] else None
        return dx, dw, None


def linear(x, weight, settings: Checkpoints):
    """x @ weight.T for x [rows, cols] in bf16 or fp16; x is kept as an 8-bit checkpoint."""
    if weight.requires_grad and torch.is_grad_enabled() and x.dtype not in (torch.bfloat16, torch.float16):
        raise ValueError(f"the weight's gradient needs x in bfloat16 or float16, not {x.dtype}")
    return _Linear.apply(x, weight, settings)


class _Silu(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, settings):
        _keep(ctx, pwlq.act8_encode(x, group=settings.group, ratio=settings.ratio))
        return torch.nn.functional.silu(x)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        saved, = _kept(ctx)
        # dy * s * (1 + x * (1 - s)) in 32 bits, rounded once: 1 + x * (1 - s) cancels near x = -1.28
        x = pwlq.act8_decode(saved)
        return torch.ops.aten.silu_backward(dy, x).to(dy.dtype), None


def silu(x, settings: Checkpoints):
    """x * sigmoid(x); x is kept as an 8-bit checkpoint."""
    return _Silu.apply(x, settings)


class _BlockNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, f, pre_weight, post_weight, gate, gate_tokens, residual_scale, eps, settings):
        r, h, saved = pwlq.block_norm(x, f, pre_weight, post_weight, gate, gate_tokens,
                                      residual_scale, eps, save=(settings.group, settings.ratio))
        _keep(ctx, saved, pre_weight, post_weight, gate)
        ctx.set_materialize_grads(False)
        return r, h

    @staticmethod
    @once_differentiable
    def backward(ctx, dr, dh):
        if dr is None and dh is None:
            return (None,) * 9
        saved, *weights = _kept(ctx)
        saved.pre_weight, saved.post_weight, saved.gate = weights
        if dh is None and saved.pre_weight is not None:
            dh = torch.zeros_like(dr)
        g = pwlq.block_norm_backward(saved, *(d.contiguous() if d is not None else None for d in (dh, dr)))
        return (g["dx"], g["df"], g["dpre"], g["dpost"], g["dgate"]) + (None,) * 4


def block_norm(x, f, pre_weight, post_weight=None, gate=None, gate_tokens=None, residual_scale=1.0,
               eps=1e-6, settings=Checkpoints()):
    """(r, h): r = residual_scale * x + gate * N(f; post_weight), h = N(r; pre_weight).  f may be None
    (the norm before the first block), and so may ``pre_weight`` (after the last one; h is None then).
    r and f are kept as 8-bit checkpoints, as far as the gradients need them."""
    return _BlockNorm.apply(x, f, pre_weight, post_weight, gate, gate_tokens, residual_scale, eps,
                            settings)
