"""What the training operators are measured on: 8-bit activation checkpoints, the weight gradient taken
from them, and the norms around a residual block, forward and backward.

``run`` gives the plain form (elementary torch operations in 32 bits) where ``own`` is false and the
library's calls where it is true.

A checkpoint holds x[T, D] as one byte per value, sign << 7 | region << 6 | level, and one binary32
range m per group of consecutive values of a row.  With p = ratio * m a byte stands for
+-level * p / 63 (region 0) or +-(p + level * (m - p) / 63) (region 1).
"""
import math

import torch

own = False

_TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
_L = 63
_TINY = 2.0 ** -100          # a range below this is held as 0
_EPS = 1e-6


# ------------------------------------------------------------------------------------- the cases
def listed():
    return [
        # one short sequence of an adapter's fine-tuning, rows of a wide model: launch latency counts
        dict(name="ckpt_16x4096_fp16", kind="ckpt", tokens=16, features=4096, dtype="fp16", group=128,
             ratio=0.5, pad=0),
        # fp32 activations of odd width, the left part of wider rows (a column slice of a fused projection)
        dict(name="ckpt_4097x2731_fp32_sliced", kind="ckpt", tokens=4097, features=2731, dtype="fp32",
             group=64, ratio=0.375, pad=37),
        # the tokens of a whole micro-batch
        dict(name="ckpt_16384x4096_bf16", kind="ckpt", tokens=16384, features=4096, dtype="bf16",
             group=128, ratio=0.4375, pad=0),
        # serving, one token: what every decoding step pays per block
        dict(name="norm_serve_1x4096_bf16", kind="serve", tokens=1, features=4096, dtype="bf16", gate=0),
        # serving, one step of many sequences, odd width, fp32, one gate for every sequence's token
        dict(name="norm_serve_97x2570_fp32", kind="serve", tokens=97, features=2570, dtype="fp32", gate=1),
        # serving, a long prompt with one gate per channel
        dict(name="norm_serve_8192x4096_bf16", kind="serve", tokens=8192, features=4096, dtype="bf16",
             gate=8192),
        # training, small model, ragged token count, one gate per channel
        dict(name="norm_train_1537x1280_fp16", kind="train", tokens=1537, features=1280, dtype="fp16",
             group=64, ratio=0.5, gate=1537),
        # training, a wide model, no gate
        dict(name="norm_train_4096x8192_bf16", kind="train", tokens=4096, features=8192, dtype="bf16",
             group=256, ratio=0.375, gate=0),
        # training, a micro-batch of eight sequences with a gate each
        dict(name="norm_train_16384x4096_bf16", kind="train", tokens=16384, features=4096, dtype="bf16",
             group=128, ratio=0.4375, gate=2048),
        # the classifier of a small network, few tokens and odd sizes, nothing aligned
        dict(name="wgrad_333x515x1283_bf16", kind="wgrad", tokens=333, outputs=515, features=1283,
             dtype="bf16", group=32, ratio=0.375, pad=1),
        # ResNet-50's classifier, 1000 x 2048: few output tiles, a long sum
        dict(name="wgrad_8192x1000x2048_fp16", kind="wgrad", tokens=8192, outputs=1000, features=2048,
             dtype="fp16", group=64, ratio=0.5, pad=0),
        # a square projection of a wide model, one micro-batch
        dict(name="wgrad_8192x4096x4096_bf16", kind="wgrad", tokens=8192, outputs=4096, features=4096,
             dtype="bf16", group=128, ratio=0.4375, pad=0),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["ckpt", "serve", "train", "wgrad"])
    group = rng.choice([32, 64, 128, 256])
    ratio = rng.choice([0.3125, 0.375, 0.4375, 0.5])

    def width(lo, hi):       # half of the widths are a multiple of 64, as models have them
        d = _log_int(rng, lo, hi)
        return max(64, d // 64 * 64) if rng.random() < 0.5 else d

    if kind == "ckpt":
        d = width(64, 16384)
        return dict(kind=kind, tokens=_log_int(rng, 1, min(65536, 16384 * 4096 // d)), features=d,
                    dtype=rng.choice(["fp32", "bf16", "fp16"]) if d <= 2048 else rng.choice(["bf16", "fp16"]),
                    group=group, ratio=ratio, pad=rng.choice([0, 0, 64, 5]))
    if kind == "serve":
        d = width(64, 12288)
        t = _log_int(rng, 1, min(16384, 8192 * 4096 // d))
        return dict(kind=kind, tokens=t, features=d,
                    dtype=rng.choice(["fp32", "bf16", "fp16"]) if d <= 2048 else rng.choice(["bf16", "fp16"]),
                    gate=rng.choice([0, 1, t, max(1, t // 3)]))
    if kind == "train":
        d = width(64, 12288)
        t = _log_int(rng, 1, min(65536, 16384 * 4096 // d))
        return dict(kind=kind, tokens=t, features=d, dtype=rng.choice(["bf16", "fp16"]), group=group,
                    ratio=ratio, gate=rng.choice([0, t, max(1, t // 5)]))
    n, k = width(64, 8192), width(64, 8192)
    most = min(32768, 8192 * 4096 * 4096 // (n * k))
    return dict(kind=kind, tokens=_log_int(rng, 1, most), outputs=n, features=k,
                dtype=rng.choice(["bf16", "fp16"]), group=group, ratio=ratio, pad=rng.choice([0, 0, 8, 3]))


# ------------------------------------------------------------------------------------ the inputs
def _rand(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)


def _activations(g, t, d):
    """Bell-shaped with long tails, a few channels several times as large as the rest."""
    x = _rand(g, t, d)
    x.mul_(1.0 + 0.25 * x.abs())
    big = torch.rand(d, generator=g, device="cuda") < 0.01
    return x.mul_(torch.where(big, 8.0, 1.0))


def _grad(g, t, d):
    return _rand(g, t, d).mul_(0.02)


def _sliced(x, pad):
    """x as the left part of rows that are `pad` values longer."""
    if not pad:
        return x
    wide = torch.empty(x.shape[0], x.shape[1] + pad, dtype=x.dtype, device=x.device)
    wide[:, :x.shape[1]] = x
    return wide[:, :x.shape[1]]


def _in_groups(x, group):
    t, d = x.shape
    n = -(-d // group)
    return torch.nn.functional.pad(x, (0, n * group - d)).view(t, n, group)


def _code(x, group, ratio):
    """(m, sign, region, level) of x in 32 bits, per group."""
    g = _in_groups(x, group)
    a = g.abs()
    m = a.amax(dim=2, keepdim=True)
    m = torch.where(m < _TINY, 0.0, m)
    m = torch.where(torch.isfinite(m), m, math.nan)
    p = m * ratio
    d = m - p
    region = a > p
    inv = torch.where(region, torch.where(d > 0, _L / d, 0.0), torch.where(p > 0, _L / p, 0.0))
    level = torch.round((a - torch.where(region, p, 0.0)) * inv).clamp(max=float(_L))
    empty = m == 0
    return m, (g < 0) & ~empty, region & ~empty, torch.where(empty, 0.0, level)


def _values(m, sign, region, level, ratio, d):
    """What (m, sign, region, level) stand for, [T, d]."""
    p = m * ratio
    v = torch.where(region, level * ((m - p) / _L) + p, level * (p / _L))
    return torch.where(sign, -v, v).flatten(1)[:, :d]


def _bytes(codes, d, group):
    """(sign, region, level) of the bytes of a checkpoint, per group."""
    c = _in_groups(codes[:, :d].to(torch.int32), group)
    return (c & 128) != 0, (c & 64) != 0, (c & 63).float()


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    kind, t, d, dt = case["kind"], case["tokens"], case["features"], _TYPES[case["dtype"]]
    s = dict(case)
    if kind == "ckpt":
        s["x"] = _sliced(_activations(g, t, d).to(dt), case["pad"])
        return s
    if kind == "wgrad":
        # the checkpoint as an encode call has left it: rows of bytes on a 16-byte pitch, and the ranges
        m, sign, region, level = _code(_activations(g, t, d).to(dt).float(), case["group"], case["ratio"])
        c = (sign.to(torch.uint8) * 128 + region.to(torch.uint8) * 64 + level.to(torch.uint8)).flatten(1)[:, :d]
        s["codes"] = torch.zeros(t, -(-d // 16) * 16, dtype=torch.uint8, device="cuda")
        s["codes"][:, :d] = c
        s["ranges"] = m[:, :, 0].contiguous()
        s["dy"] = _sliced(_grad(g, t, case["outputs"]).to(dt), case["pad"])
        return s
    s["x"] = _activations(g, t, d).to(dt)
    s["f"] = _activations(g, t, d).mul_(0.3).to(dt)
    s["pre"] = (1.0 + 0.1 * _rand(g, d)).to(dt)
    s["post"] = (1.0 + 0.1 * _rand(g, d)).to(dt)
    every = case["gate"]
    s["gates"] = (0.5 + 0.3 * _rand(g, -(-t // every), d)).to(dt) if every else None
    s["scale"] = 0.75
    if kind == "train":
        s["dh"] = _grad(g, t, d).to(dt)
        s["dr"] = _grad(g, t, d).to(dt)
    return s


# ------------------------------------------------------------------------------------- the passes
def run(state):
    return (_RUN_OWN if own else _RUN_PLAIN)[state["kind"]](state)


def _plain_ckpt(s):
    v = _values(*_code(s["x"].float(), s["group"], s["ratio"]), s["ratio"], s["features"])
    return {"x": v.to(s["x"].dtype)}


def _own_ckpt(s):
    from paper_2002_00104_b200 import pwlq
    saved = pwlq.act8_encode(s["x"], group=s["group"], ratio=s["ratio"])
    return {"x": pwlq.act8_decode(saved, dtype=s["x"].dtype)}


def _gate_rows(s):
    """The gates of every token, [T, D]."""
    if s["gates"] is None:
        return torch.ones((), device="cuda")
    at = torch.arange(s["tokens"], device="cuda") // s["gate"]
    return s["gates"].float()[at]


def _rstd(v):
    return torch.rsqrt((v * v).mean(dim=1, keepdim=True) + _EPS)


def _plain_forward(s):
    x, f = s["x"].float(), s["f"].float()
    rf = _rstd(f)
    r = s["scale"] * x + _gate_rows(s) * (f * rf * s["post"].float())
    rr = _rstd(r)
    return r, r * rr * s["pre"].float(), rf, rr


def _plain_serve(s):
    r, h, _, _ = _plain_forward(s)
    return {"r": r.to(s["x"].dtype), "h": h.to(s["x"].dtype)}


def _own_serve(s):
    from paper_2002_00104_b200 import pwlq
    r, h, _ = pwlq.block_norm(s["x"], s["f"], pre_weight=s["pre"], post_weight=s["post"], gate=s["gates"],
                              gate_tokens=s["gate"], residual_scale=s["scale"], eps=_EPS)
    return {"r": r, "h": h}


def _plain_train(s):
    r, h, rf, rr = _plain_forward(s)
    group, ratio, d, dt = s["group"], s["ratio"], s["features"], s["x"].dtype
    n_r = _values(*_code(r, group, ratio), ratio, d) * rr
    n_f = _values(*_code(s["f"].float(), group, ratio), ratio, d) * rf
    dh, post, gate = s["dh"].float(), s["post"].float(), _gate_rows(s)
    u = dh * s["pre"].float()
    dres = s["dr"].float() + rr * (u - n_r * (u * n_r).mean(dim=1, keepdim=True))
    do = dres * gate
    v = do * post
    df = rf * (v - n_f * (v * n_f).mean(dim=1, keepdim=True))
    out = {"r": r.to(dt), "h": h.to(dt), "dx": (s["scale"] * dres).to(dt), "df": df.to(dt),
           "dpre": (dh * n_r).sum(dim=0).to(dt), "dpost": (do * n_f).sum(dim=0).to(dt)}
    if s["gates"] is not None:
        at = torch.arange(s["tokens"], device="cuda") // s["gate"]
        dgate = torch.zeros(s["gates"].shape, dtype=torch.float32, device="cuda")
        out["dgate"] = dgate.index_add_(0, at, dres * n_f * post).to(dt)
    return out


def _own_train(s):
    from paper_2002_00104_b200 import pwlq
    r, h, saved = pwlq.block_norm(s["x"], s["f"], pre_weight=s["pre"], post_weight=s["post"],
                                  gate=s["gates"], gate_tokens=s["gate"], residual_scale=s["scale"],
                                  eps=_EPS, save=(s["group"], s["ratio"]))
    grads = pwlq.block_norm_backward(saved, s["dh"], s["dr"])
    out = {"r": r, "h": h}
    out.update((k, v) for k, v in grads.items() if v is not None)
    return out


def _plain_wgrad(s):
    sign, region, level = _bytes(s["codes"], s["features"], s["group"])
    x = _values(s["ranges"].unsqueeze(2), sign, region, level, s["ratio"], s["features"])
    return {"dw": (s["dy"].float().t() @ x).to(s["dy"].dtype)}


def _own_wgrad(s):
    from paper_2002_00104_b200 import pwlq
    saved = pwlq.Act8(s["codes"], s["ranges"], s["features"], s["group"], s["ratio"])
    return {"dw": pwlq.act8_weight_grad(s["dy"], saved)}


_RUN_PLAIN = {"ckpt": _plain_ckpt, "serve": _plain_serve, "train": _plain_train, "wgrad": _plain_wgrad}
_RUN_OWN = {"ckpt": _own_ckpt, "serve": _own_serve, "train": _own_train, "wgrad": _own_wgrad}


# --------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    t, d, size = case["tokens"], case["features"], 4 if case["dtype"] == "fp32" else 2
    kind, every = case["kind"], case.get("gate", 0)
    ranges = 4 * t * -(-d // case["group"]) if "group" in case else 0
    small = size * d * (2 + (-(-t // every) if every else 0))          # the norms' weights and the gates
    if kind == "ckpt":       # values in, bytes and ranges out; bytes and ranges in, values out
        return {"bytes": t * d * (2 * size + 2) + 2 * ranges, "flops": 20 * t * d}
    if kind == "serve":      # x, f in; r, h out
        return {"bytes": 4 * size * t * d + small, "flops": 12 * t * d}
    if kind == "train":      # the same, two checkpoints out and in, dh, dr in, dx, df out
        return {"bytes": 8 * size * t * d + 2 * (2 * t * d + 2 * ranges) + 16 * t + 3 * small,
                "flops": 70 * t * d}
    n = case["outputs"]
    return {"bytes": size * t * n + t * d + ranges + size * n * d, "flops": 2 * t * n * d}


# ------------------------------------------------------------------------------------ in 64 bits
def _exact_held(x, group, ratio):
    """The real number that a checkpoint holds for every value of x (binary64 throughout)."""
    t, d = x.shape
    n = (d + group - 1) // group
    y = torch.zeros(t, n * group, dtype=torch.float64, device=x.device)
    y[:, :d] = x
    y = y.view(t, n, group)
    m = y.abs().max(dim=2).values.unsqueeze(2)
    m = m * (m >= _TINY)
    p = ratio * m
    one = torch.ones_like(m)
    center = torch.minimum(y.abs(), p) / torch.where(p > 0, p, one)      # 0..1 along [0, p]
    tail = (y.abs() - p).clamp(min=0) / torch.where(m > p, m - p, one)   # 0..1 along [p, m]
    v = torch.where(y.abs() > p, p + (m - p) * (torch.round(tail * _L) / _L), p * (torch.round(center * _L) / _L))
    return (v * torch.sign(y)).reshape(t, n * group)[:, :d]


def exact(case, seed):
    s = prepare(case, seed)
    kind, d = case["kind"], case["features"]
    if kind == "ckpt":
        return {"x": _exact_held(s["x"].double(), s["group"], s["ratio"])}
    if kind == "wgrad":
        c = s["codes"][:, :d].long()
        m = s["ranges"].double().repeat_interleave(s["group"], dim=1)[:, :d]
        step = (c % 64).double() / _L
        x = torch.where((c // 64) % 2 == 1, m * (s["ratio"] + (1 - s["ratio"]) * step), m * s["ratio"] * step)
        x = x * (1 - 2 * (c // 128)).double()
        return {"dw": torch.einsum("tn,tk->nk", s["dy"].double(), x)}
    x, f, pre, post = (s[k].double() for k in ("x", "f", "pre", "post"))
    t = x.shape[0]
    if s["gates"] is None:
        gate = torch.ones(t, 1, dtype=torch.float64, device="cuda")
    else:
        gate = s["gates"].double().repeat_interleave(s["gate"], dim=0)[:t]
    sf = 1.0 / (f.square().sum(1, keepdim=True) / d + _EPS).sqrt()
    r = s["scale"] * x + gate * post * f * sf
    sr = 1.0 / (r.square().sum(1, keepdim=True) / d + _EPS).sqrt()
    out = {"r": r, "h": pre * r * sr}
    if kind == "serve":
        return out
    nr = _exact_held(r, s["group"], s["ratio"]) * sr
    nf = _exact_held(f, s["group"], s["ratio"]) * sf
    dh = s["dh"].double()
    c = (dh * pre * nr).sum(1, keepdim=True) / d
    e = s["dr"].double() + sr * dh * pre - sr * nr * c
    w = e * gate * post
    out["dx"] = s["scale"] * e
    out["df"] = sf * w - sf * nf * ((w * nf).sum(1, keepdim=True) / d)
    out["dpre"] = (dh * nr).sum(0)
    out["dpost"] = (e * gate * nf).sum(0)
    if s["gates"] is not None:
        b = s["gates"].shape[0]
        z = torch.zeros(b * s["gate"], d, dtype=torch.float64, device="cuda")
        z[:t] = e * nf * post
        out["dgate"] = z.view(b, s["gate"], d).sum(1)
    return out
