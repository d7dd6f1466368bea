"""Plain forms of the training operators for their tests: bytes and values of 8-bit checkpoints in
binary32 by NumPy, norms and gradients in binary64 by torch."""
import numpy as np
import torch

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
# largest relative rounding to the type (half of its eps); and half the smallest subnormal
HALF_ULP = {t: torch.finfo(t).eps / 2 for t in (torch.float32, torch.bfloat16, torch.float16)}
SUBNORMAL = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}
U = 2.0 ** -24                                   # unit roundoff of binary32
TINY = 2.0 ** -100


def in_groups(x, group):
    rows, cols = x.shape
    n = -(-cols // group)
    y = np.zeros((rows, n * group), x.dtype)
    y[:, :cols] = x
    return y.reshape(rows, n, group)


def act8_reference(x, group, ratio):
    """(bytes [rows, cols], ranges [rows, groups], values [rows, cols]) of binary32 x: the format's
    sequence, one NumPy binary32 operation at a time."""
    rows, cols = x.shape
    one, levels = np.float32(1), np.float32(63)
    g = in_groups(x.astype(np.float32), group)
    with np.errstate(all="ignore"):
        m = np.abs(g).max(axis=2, keepdims=True)     # NaN wins
        m = np.where(np.isfinite(m), m, np.float32("nan"))
        m = np.where(m < np.float32(TINY), np.float32(0), m)
        p = m * np.float32(ratio)
        d = m - p
        s1, s2 = p * (one / levels), d * (one / levels)
        inv1 = np.where(p > 0, one / p * levels, np.float32(0))
        inv2 = np.where(d > 0, one / d * levels, np.float32(0))
        a = np.abs(g)
        tail = a > p
        t = (a - np.where(tail, p, np.float32(0))) * np.where(tail, inv2, inv1)
        q = np.minimum(np.rint(t), levels)
        v = np.where(tail, q * s2 + p, q * s1)
    held = m > 0
    q = np.where(held, q, 0).astype(np.uint8)
    neg = (g < 0) & held
    b = neg.astype(np.uint8) << 7 | (tail & held).astype(np.uint8) << 6 | q
    v = np.where(held, np.where(neg, -v, v), m)       # 0 and NaN stand for themselves
    assert v.dtype == m.dtype == np.float32
    return b.reshape(rows, -1)[:, :cols], m[:, :, 0], v.reshape(rows, -1)[:, :cols]


def act8_values64(codes, ranges, cols, group, ratio):
    """What the bytes of a checkpoint stand for, in binary64 (torch tensors in and out)."""
    c = codes[:, :cols].long()
    m = ranges.double().repeat_interleave(group, dim=1)[:, :cols]
    p = (ranges * torch.tensor(ratio, dtype=torch.float32, device=ranges.device)).double()
    p = p.repeat_interleave(group, dim=1)[:, :cols]
    q = (c & 63).double() / 63.0
    v = torch.where((c & 64) != 0, p + q * (m - p), q * p)
    return torch.where((c & 128) != 0, -v, v)


def held64(saved):
    return act8_values64(saved.codes, saved.ranges, saved.cols, saved.group, saved.ratio)


def on_grid(rng, rows, cols, group, step):
    """Values that a checkpoint at ratio 0.5 holds exactly: multiples of `step` up to 126, one of
    which is 126 in every group."""
    x = rng.integers(-100, 101, (rows, cols)).astype(np.float64)
    x[:, ::group] = 126.0 * rng.choice([-1.0, 1.0], x[:, ::group].shape)
    return x * step


def rstd(v, eps):
    return (v.square().mean(dim=1, keepdim=True) + eps).rsqrt()


def gate_rows(gate, every, rows):
    return gate.repeat_interleave(every, dim=0)[:rows]


def forward64(x, f, pre, post, gate, every, scale, eps, offset):
    """(r, h, rstd_r, rstd_f) in binary64."""
    r = scale * x
    rf = None
    if f is not None:
        o = f
        if post is not None:
            rf = rstd(f, eps)
            o = f * rf * (post + offset)
        if gate is not None:
            o = o * gate_rows(gate, every, x.shape[0])
        r = r + o
    if pre is None:
        return r, None, None, rf
    rr = rstd(r, eps)
    return r, r * rr * (pre + offset), rr, rf


def backward64(R, F, rr, rf, dh, dr, pre, post, gate, every, scale, offset, has_f=True):
    """Gradients in binary64 at the checkpoints' values R, F, and for each of them the sum of the
    magnitudes that its binary32 evaluation adds up (what rounding errors are proportional to)."""
    zero = torch.zeros_like(dh if dh is not None else dr)
    e, size = zero, zero
    if pre is not None:
        n = R * rr
        u = dh * (pre + offset)
        c, ca = (u * n).mean(1, keepdim=True), (u * n).abs().mean(1, keepdim=True)
        e = rr * (u - n * c)
        size = rr * (u.abs() + n.abs() * ca)
    if dr is not None:
        e = e + dr
        size = size + dr.abs()
    out = {"dx": scale * e}
    mag = {"dx": abs(scale) * size}
    if pre is not None:
        out["dpre"], mag["dpre"] = (dh * n).sum(0), (dh * n).abs().sum(0)
    if not has_f:
        return out, mag
    g = gate_rows(gate, every, zero.shape[0]) if gate is not None else torch.ones_like(zero)
    w = post + offset if post is not None else torch.ones_like(zero[0])
    v, vs = e * g * w, size * (g * w).abs()
    if post is None:
        n = F
        out["df"], mag["df"] = v, vs
    else:
        n = F * rf
        c, ca = (v * n).mean(1, keepdim=True), (vs * n.abs()).mean(1, keepdim=True)
        out["df"] = rf * (v - n * c)
        mag["df"] = rf * (vs + n.abs() * ca)
        out["dpost"], mag["dpost"] = (e * g * n).sum(0), (size * (g * n).abs()).sum(0)
    if gate is not None:
        k = gate.shape[0]
        for d, src in ((out, e * n * w), (mag, size * (n * w).abs())):
            z = torch.zeros(k * every, zero.shape[1], dtype=torch.float64, device=zero.device)
            z[:zero.shape[0]] = src
            d["dgate"] = z.view(k, every, -1).sum(1)
    return out, mag


def check(got, want, extra, what):
    """|got - want| <= half an ulp of got's type at want, and `extra` (what binary32 may be off)."""
    dt = got.dtype
    diff = (got.double() - want).abs()
    # an error of `extra` can also move the rounding itself by as much
    bound = HALF_ULP[dt] * want.abs() + SUBNORMAL[dt] + extra * (1 + HALF_ULP[dt])
    bad = ~(diff <= bound)
    assert not bad.any(), (f"{what}: {int(bad.sum())} of {bad.numel()} off, worst "
                           f"{float((diff / bound).nan_to_num(nan=1e30).max()):.3g} of the bound")
