"""What the operators on 4-bit weights are measured on: packing a weight matrix, its product with a few
tokens, and a whole mixture-of-experts layer for a few tokens.

``run`` gives the plain form (elementary torch operations in 32 bits, the router's scores in 64) where
``own`` is false and the library's calls where it is true.

A row of a weight matrix is cut into groups of consecutive values with one bfloat16 scale s each.  A value is
sign, region and a level q of 0..3, and stands for +-n * s with n = q * b in the center (region 0) and
n = 3 * b + q * (64 - b) in the tail (region 1): the two-piece quantizer whose range is m = 192 * s and whose
breakpoint is p = m * b / 64, b = 64 * ratio a whole number.
"""
import math

import torch

own = False

_TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
_TINY = 2.0 ** -100          # a range below this is held as 0


# ------------------------------------------------------------------------------------- the cases
def listed():
    return [
        # ResNet-50's classifier, 1000 x 2048, quantized once when the model is loaded
        dict(name="pack_1000x2048_fp32", kind="pack", outputs=1000, features=2048, dtype="fp32", group=64,
             ratio=0.4375, pad=0),
        # one large projection of a model that is being loaded
        dict(name="pack_8192x8192_bf16", kind="pack", outputs=8192, features=8192, dtype="bf16", group=128,
             ratio=0.421875, pad=0),
        # the same classifier on one image's features: launch latency counts
        dict(name="linear_1x1000x2048_fp32", kind="linear", tokens=1, outputs=1000, features=2048, dtype="fp32",
             group=64, ratio=0.4375, paired=False, pad=0),
        # one token through a square projection: the ordinary decoding step
        dict(name="linear_1x4096x4096_bf16", kind="linear", tokens=1, outputs=4096, features=4096, dtype="bf16",
             group=128, ratio=0.421875, paired=False, pad=0),
        # one token through gate and up projection of a wide model, with the activation between them
        dict(name="gated_1x22528x8192_bf16", kind="linear", tokens=1, outputs=22528, features=8192, dtype="bf16",
             group=128, ratio=0.421875, paired=True, pad=0),
        # a few sequences, odd sizes, the left part of wider rows, nothing aligned
        dict(name="linear_7x2731x1285_fp16", kind="linear", tokens=7, outputs=2731, features=1285, dtype="fp16",
             group=32, ratio=0.5, paired=False, pad=3),
        # a batch of sequences, one step, a large projection
        dict(name="linear_16x8192x8192_bf16", kind="linear", tokens=16, outputs=8192, features=8192, dtype="bf16",
             group=128, ratio=0.421875, paired=False, pad=0),
        # a full batch, gate and up projection
        dict(name="gated_64x16384x4096_fp16", kind="linear", tokens=64, outputs=16384, features=4096, dtype="fp16",
             group=64, ratio=0.375, paired=True, pad=0),
        # one token, many small experts of which few are chosen
        dict(name="moe_1x2048_64of8_bf16", kind="moe", tokens=1, features=2048, hidden=1024, experts=64, top=8,
             dtype="bf16", group=128, ratio=0.421875, normalize=True),
        # a few sequences, few large experts
        dict(name="moe_4x4096_8of2_fp16", kind="moe", tokens=4, features=4096, hidden=8192, experts=8, top=2,
             dtype="fp16", group=128, ratio=0.421875, normalize=True),
        # odd sizes, fp32, weights of the chosen experts as they come out of the softmax over all
        dict(name="moe_5x1287_17of3_fp32", kind="moe", tokens=5, features=1287, hidden=515, experts=17, top=3,
             dtype="fp32", group=32, ratio=0.5, normalize=False),
        # a full batch over many small experts: nearly every expert is read
        dict(name="moe_64x2048_128of8_bf16", kind="moe", tokens=64, features=2048, hidden=768, experts=128, top=8,
             dtype="bf16", group=64, ratio=0.4375, normalize=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["pack", "linear", "linear", "moe"])
    dtype = rng.choice(["fp32", "bf16", "bf16", "fp16", "fp16"])
    group = rng.choice([32, 64, 128, 256])
    ratio = rng.choice([20, 24, 27, 28, 32]) / 64

    def width(lo, hi):       # half of the widths are a multiple of 64, as models have them
        d = _log_int(rng, lo, hi)
        return max(64, d // 64 * 64) if rng.random() < 0.5 else d

    if kind == "pack":
        n = width(64, 16384)
        return dict(kind=kind, outputs=n, features=width(64, min(16384, 8192 * 8192 // n)), dtype=dtype, group=group,
                    ratio=ratio, pad=rng.choice([0, 0, 64, 5]))
    if kind == "linear":
        paired = rng.random() < 0.4
        n = width(64, 22528)
        n -= n % 2 if paired else 0
        k = width(64, min(16384, 22528 * 8192 // n))
        return dict(kind=kind, tokens=_log_int(rng, 1, 64), outputs=n, features=k, dtype=dtype, group=group,
                    ratio=ratio, paired=paired, pad=rng.choice([0, 0, 8, 3]))
    e = rng.choice([4, 8, 17, 32, 64, 128])
    d = width(64, 4096)
    f = width(64, min(8192, 8 * 4096 * 8192 // (e * d)))
    return dict(kind=kind, tokens=_log_int(rng, 1, 64), features=d, hidden=f, experts=e,
                top=rng.randint(1, min(8, e)), dtype=dtype, group=group, ratio=ratio,
                normalize=rng.random() < 0.7)


# ------------------------------------------------------------------------------------ the inputs
def _rand(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)


def _weights(g, n, k, dtype):
    """Bell-shaped with long tails, rows of different size, of such a norm that products keep theirs."""
    w = _rand(g, n, k)
    w.mul_(1.0 + 0.25 * w.abs()).mul_(0.7 * k ** -0.5)
    return w.mul_(0.5 + torch.rand(n, 1, generator=g, device="cuda")).to(dtype)


def _activations(g, t, d):
    """Bell-shaped with long tails, a few channels several times as large as the rest."""
    x = _rand(g, t, d)
    x.mul_(1.0 + 0.25 * x.abs())
    big = torch.rand(d, generator=g, device="cuda") < 0.01
    return x.mul_(torch.where(big, 8.0, 1.0))


def _sliced(x, pad):
    """x as the left part of rows that are `pad` values longer."""
    if not pad:
        return x
    wide = torch.empty(x.shape[0], x.shape[1] + pad, dtype=x.dtype, device=x.device)
    wide[:, :x.shape[1]] = x
    return wide[:, :x.shape[1]]


def _raw(case, seed):
    """Weights as the model has them, and the tokens."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt, kind, d = _TYPES[case["dtype"]], case["kind"], case["features"]
    s = dict(case)
    if kind == "pack":
        s["w"] = _sliced(_weights(g, case["outputs"], d, dt), case["pad"])
        return s
    t = case["tokens"]
    if kind == "linear":
        s["w"] = _weights(g, case["outputs"], d, dt)
        s["x"] = _sliced(_activations(g, t, d).to(dt), case["pad"])
        return s
    e, f = case["experts"], case["hidden"]
    s["w_up"] = _weights(g, e * 2 * f, d, dt).view(e, 2 * f, d)        # gate rows, then up rows
    s["w_down"] = _weights(g, e * d, f, dt).view(e, d, f)
    s["router"] = (_rand(g, e, d) * 1.5 * d ** -0.5).to(dt)
    s["x"] = _activations(g, t, d).to(dt)
    return s


def prepare(case, seed):
    s = _raw(case, seed)
    packed = {"pack": [], "linear": ["w"], "moe": ["w_up", "w_down"]}[case["kind"]]
    # a program that serves keeps its weights packed: each form in the layout that it reads
    for name in packed:
        w = s.pop(name)
        if own:
            from paper_2002_00104_b200 import pwlq
            paired = case["kind"] == "moe" and name == "w_up" or case.get("paired", False)
            s[name] = pwlq.w4_encode(w, group=case["group"], ratio=case["ratio"], paired=paired)
        else:
            s[name] = _pack(w, case["group"], case["ratio"])
    return s


# ------------------------------------------------------------------------------------- the passes
def run(state):
    return (_RUN_OWN if own else _RUN_PLAIN)[state["kind"]](state)


def _in_groups(w, group):
    n = -(-w.shape[-1] // group)
    return torch.nn.functional.pad(w, (0, n * group - w.shape[-1])).unflatten(-1, (n, group))


def _scales(w, group):
    """The groups' scales, in 32 bits."""
    m = _in_groups(w, group).abs().amax(dim=-1)
    m = torch.where(m < _TINY, 0.0, m)
    bits = (m / 192.0).view(torch.int32)
    return torch.where(torch.isfinite(m), ((bits + 0xFFFF) & -0x10000).view(torch.float32), math.nan)


def _levels(w, s, group, ratio):
    """(sign, region, level) per group; a product of a scale and a bound is exact in 32 bits."""
    b = round(64 * ratio)
    a, s = _in_groups(w, group), s.unsqueeze(-1)
    sign, a = a < 0, a.abs()
    region = a > 3.0 * b * s
    z = torch.where(region, 3.0 * b, 0.0)
    step = torch.where(region, 64.0 - b, 1.0 * b)
    # halves go to the even level
    q = ((a > (z + 0.5 * step) * s).to(torch.uint8) + (a >= (z + 1.5 * step) * s).to(torch.uint8)
         + (a > (z + 2.5 * step) * s).to(torch.uint8))
    empty = ~(s > 0)
    return sign & ~empty, region & ~empty, torch.where(empty, 0, q)


def _multiples(sign, region, q, ratio):
    b = 64.0 * ratio
    n = torch.where(region, 3.0 * b + q * (64.0 - b), q * b)
    return torch.where(sign, -n, n)


def _pack(w, group, ratio):
    """(two values a byte [..., n, groups, group / 2], scales [..., n, groups]) of a weight tensor."""
    parts, scales = [], []
    for part in w.flatten(0, -2).split(16384):
        v = part.float()
        s = _scales(v, group)
        sign, region, q = _levels(v, s, group, ratio)
        c = sign.to(torch.uint8) * 8 + region.to(torch.uint8) * 4 + q
        parts.append(c[..., ::2] + 16 * c[..., 1::2])
        scales.append(s.bfloat16())
    codes, s = torch.cat(parts), torch.cat(scales)
    return codes.view(*w.shape[:-1], *codes.shape[1:]), s.view(*w.shape[:-1], s.shape[1])


def _unpack(packed, features, ratio):
    codes, s = packed
    c = torch.stack((codes & 15, codes >> 4), dim=-1).flatten(-2)
    v = _multiples((c & 8) != 0, (c & 4) != 0, (c & 3).float(), ratio) * s.float().unsqueeze(-1)
    return v.flatten(-2)[..., :features]


def _plain_pack(s):
    w = s["w"].float()
    scale = _scales(w, s["group"])
    v = _multiples(*_levels(w, scale, s["group"], s["ratio"]), s["ratio"]) * scale.unsqueeze(-1)
    return {"values": v.flatten(1)[:, :s["features"]].to(s["w"].dtype)}


def _own_pack(s):
    from paper_2002_00104_b200 import pwlq
    packed = pwlq.w4_encode(s["w"], group=s["group"], ratio=s["ratio"])
    return {"values": pwlq.w4_decode(packed, dtype=s["w"].dtype)}


def _gated(v):
    gate, up = v.chunk(2, dim=-1)
    return gate / (1.0 + torch.exp(-gate)) * up


def _plain_linear(s):
    y = s["x"].float() @ _unpack(s["w"], s["features"], s["ratio"]).t()
    return {"y": (_gated(y) if s["paired"] else y).to(s["x"].dtype)}


def _own_linear(s):
    from paper_2002_00104_b200 import pwlq
    return {"y": pwlq.w4_linear(s["x"], s["w"])}


def _plain_moe(s):
    x, k, e = s["x"].float(), s["top"], s["experts"]
    # 64 bits: two experts' scores may lie next to each other
    scores = s["x"].double() @ s["router"].double().t()
    order = torch.sort(scores, dim=1, descending=True, stable=True)
    chosen, best = order.indices[:, :k], order.values[:, :k]
    over = best if s["normalize"] else scores
    top = best[:, :1]
    weight = (torch.exp(best - top) / torch.exp(over - top).sum(dim=1, keepdim=True)).float()
    if s["tokens"] * k < e:                       # the chosen experts' weights alone, one copy for each token
        up = _unpack(tuple(v[chosen.flatten()] for v in s["w_up"]), s["features"], s["ratio"])
        down = _unpack(tuple(v[chosen.flatten()] for v in s["w_down"]), s["hidden"], s["ratio"])
        h = _gated(torch.bmm(up, x.repeat_interleave(k, dim=0).unsqueeze(2)).squeeze(2)) * weight.view(-1, 1)
        y = torch.bmm(down, h.unsqueeze(2)).view(s["tokens"], k, -1).sum(dim=1)
    else:                                         # every expert for every token, and weight 0 where not chosen
        up = _unpack(s["w_up"], s["features"], s["ratio"])
        h = _gated(torch.matmul(x, up.transpose(1, 2)))
        h = h * torch.zeros_like(scores, dtype=torch.float32).scatter_(1, chosen, weight).t().unsqueeze(2)
        del up
        y = torch.bmm(h, _unpack(s["w_down"], s["hidden"], s["ratio"]).transpose(1, 2)).sum(dim=0)
    return {"y": y.to(s["x"].dtype), "experts": chosen.int(), "weights": weight}


def _own_moe(s):
    from paper_2002_00104_b200 import pwlq
    y, experts, weights = pwlq.w4_moe(s["x"], s["router"], s["w_up"], s["w_down"], s["top"],
                                      normalize=s["normalize"], want_routing=True)
    return {"y": y, "experts": experts, "weights": weights}


_RUN_PLAIN = {"pack": _plain_pack, "linear": _plain_linear, "moe": _plain_moe}
_RUN_OWN = {"pack": _own_pack, "linear": _own_linear, "moe": _own_moe}


# --------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    d, size, group = case["features"], 4 if case["dtype"] == "fp32" else 2, case["group"]

    def held(n, k):          # a packed matrix: half a byte a value, two bytes a group
        return n * k // 2 + 2 * n * -(-k // group)

    if case["kind"] == "pack":       # values in, codes and scales out; codes and scales in, values out
        n = case["outputs"]
        return {"bytes": 2 * size * n * d + 2 * held(n, d), "flops": 16 * n * d}
    t = case["tokens"]
    if case["kind"] == "linear":
        n = case["outputs"]
        return {"bytes": held(n, d) + size * t * (d + (n // 2 if case["paired"] else n)), "flops": 2 * t * n * d}
    e, f, k = case["experts"], case["hidden"], case["top"]
    read = e * (1 - (1 - k / e) ** t)            # experts that t tokens choose, if all are as likely
    return {"bytes": int(read * (held(2 * f, d) + held(d, f))) + size * (e * d + 2 * t * d) + 8 * t * k,
            "flops": 2 * t * (e * d + 3 * k * d * f)}


# ------------------------------------------------------------------------------------ in 64 bits
def _exact_held(w, group, ratio):
    """The real numbers that a packed matrix holds for w [n, k]: on each piece of the range the nearest of
    four equally spaced points (binary64; the scale as the format defines it)."""
    n, k = w.shape
    groups = (k + group - 1) // group
    v = torch.zeros(n, groups * group, dtype=torch.float64, device=w.device)
    v[:, :k] = w
    v = v.view(n, groups, group)
    m = v.abs().max(dim=2).values
    s32 = (m * (m >= _TINY)).float() / torch.tensor(192.0, device=w.device)
    near = s32.bfloat16()                         # the nearest, then the next one up where that is below
    below = near.float() < s32
    s = torch.where(below, (near.view(torch.int16) + 1).view(torch.bfloat16), near).double().unsqueeze(2)
    m, p = 192 * s, 192 * s * ratio
    one = torch.ones_like(m)
    a = v.abs()
    center = p / 3 * torch.round(3 * (a / torch.where(p > 0, p, one))).clamp(max=3)
    tail = p + (m - p) / 3 * torch.round(3 * ((a - p) / torch.where(m > p, m - p, one))).clamp(min=0, max=3)
    return (torch.where(a > p, tail, center) * torch.sign(v)).reshape(n, groups * group)[:, :k]


def exact(case, seed):
    s = _raw(case, seed)
    group, ratio = case["group"], case["ratio"]
    if case["kind"] == "pack":
        return {"values": _exact_held(s["w"].double(), group, ratio)}
    x = s["x"].double()
    t = x.shape[0]
    if case["kind"] == "linear":
        out = torch.cat([x @ _exact_held(w.double(), group, ratio).t() for w in s["w"].split(4096)], dim=1)
        if case["paired"]:
            half = out.shape[1] // 2
            out = out[:, :half] * torch.sigmoid(out[:, :half]) * out[:, half:]
        return {"y": out}
    e, f, k = case["experts"], case["hidden"], case["top"]
    scores = torch.einsum("td,ed->te", x, s["router"].double())
    # the k-th place of an expert: how many are before it
    before = (scores[:, None, :] > scores[:, :, None]).sum(2)
    lower = torch.arange(e, device=x.device)[None, :] < torch.arange(e, device=x.device)[:, None]
    before = before + ((scores[:, None, :] == scores[:, :, None]) & lower).sum(2)
    share = torch.softmax(scores, dim=1)
    if case["normalize"]:
        share = share / torch.where(before < k, share, torch.zeros_like(share)).sum(1, keepdim=True)
    y = torch.zeros(t, x.shape[1], dtype=torch.float64, device=x.device)
    experts = torch.argsort(before, dim=1)[:, :k]
    for i in range(e):
        who = (before[:, i] < k).nonzero().flatten()
        if len(who):
            a = x[who] @ _exact_held(s["w_up"][i].double(), group, ratio).t()
            h = a[:, :f] * torch.sigmoid(a[:, :f]) * a[:, f:] * share[who, i:i + 1]
            y[who] += h @ _exact_held(s["w_down"][i].double(), group, ratio).t()
    return {"y": y, "experts": experts.int(), "weights": share.gather(1, experts)}
