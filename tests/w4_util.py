"""Plain forms of the operators on 4-bit weights for their tests, in binary64, and the layout of a packed matrix."""
import numpy as np
import torch

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
HALF_ULP = {t: torch.finfo(t).eps / 2 for t in TYPES.values()}
TINY = 2.0 ** -100
# A product's sum over a group is made by matrix instructions of 16 products and the sum so far, each kept to 24
# bits below the largest of the 17 or better: at most 17 * 2^-23 of the magnitudes' sum each, 8 of them to 128 columns.
# Groups (a few thousand at most) are added in binary32: 2^-24 each, random, below 64 * 2^-24.
SUM = 8 * 17 * 2.0 ** -23 + 64 * 2.0 ** -24


def scales(w, group):
    """[n, groups] of binary32 w [n, k]: max / 192 in binary32, rounded up to bfloat16."""
    n, k = w.shape
    groups = -(-k // group)
    a = torch.zeros(n, groups * group)
    a[:, :k] = w.float().abs()
    m = a.view(n, groups, group).amax(2)
    m = torch.where(m < TINY, 0.0, m)
    bits = (m / 192.0).numpy().view(np.int32).astype(np.int64)
    s = torch.from_numpy(((bits + 0xFFFF) & ~0xFFFF).astype(np.int32).view(np.float32))
    return torch.where(torch.isfinite(m), s, float("nan"))


def codes(w, group, ratio):
    """(scales, codes) of w [n, k]: sign << 3 | region << 2 | level, 0 where the value is held as 0; decided in
    binary64."""
    n, k = w.shape
    s = scales(w, group)
    b = ratio * 64
    each = s.double().repeat_interleave(group, 1)[:, :k]
    tail = w.double().abs() > 3 * b * each
    step = torch.where(tail, 64 - b, b)
    z = torch.where(tail, 3 * b, 0.0)
    x = w.double().abs()
    q = ((x > (z + 0.5 * step) * each).long() + (x >= (z + 1.5 * step) * each).long()
         + (x > (z + 2.5 * step) * each).long())
    c = tail.long() * 4 + q
    c = torch.where(c > 0, (w < 0).long() * 8 + c, 0)
    return s, torch.where(each > 0, c, 0)


def values(s, c, group, ratio):
    """What codes stand for, binary64."""
    b = ratio * 64
    q, tail = (c & 3).double(), (c & 4) != 0
    n = torch.where(tail, 3 * b + q * (64 - b), q * b)
    n = torch.where((c & 8) != 0, -n, n)
    return n * s.double().repeat_interleave(group, 1)[:, :c.shape[1]]


def held(w, group, ratio):
    """The values that w [n, k] or [e, n, k] is held as, binary64, on the CPU."""
    flat = w.cpu().flatten(0, -2)
    s, c = codes(flat, group, ratio)
    return values(s, c, group, ratio).view(w.shape)


def layout(s, c, group, paired):
    """The bytes of a packed matrix, from the format's description."""
    n, k = c.shape
    rows = [[t * 8 + r if r < 8 else n // 2 + t * 8 + r - 8 for r in range(16)] for t in range(-(-(n // 2) // 8))] \
        if paired else [[t * 16 + r for r in range(16)] for t in range(-(-n // 16))]
    half = n // 2
    out = []
    ends = 4 if group == 32 else 2 if group == 64 else 1
    bits16 = (s.numpy().view(np.int32) >> 16) & 0xFFFF
    bits16[~np.isfinite(s.numpy())] = 0x7FC0
    for tile in rows:
        def row(r):
            i = tile[r]
            if paired and (i >= half if r < 8 else i >= n):
                return None
            return i if i < n else None
        for block in range(-(-k // 128)):
            words = np.zeros((2, 32, 4), np.uint32)
            for lane in range(32):
                g, q = lane // 4, lane % 4
                for j in range(8):
                    word = 0
                    first = block * 128 + 32 * (j // 2) + 8 * q + 4 * (j % 2)
                    for side in range(2):
                        i = row(g + 8 * side)
                        for e in range(4):
                            v = int(c[i, first + e]) if i is not None and first + e < k else 0
                            word |= (v & 7) << (16 * side + 4 * e)
                            if v & 8:
                                word |= 1 << (8 * e + 7 if side == 0 else 8 * e + 3)
                    words[j // 4, lane, j % 4] = word
            scale = np.zeros((ends, 8, 2), np.uint16)
            for e in range(ends):
                at = (block * 128 + e * (128 // ends)) // group
                for r in range(16):
                    i = row(r)
                    if i is not None and at < bits16.shape[1]:
                        scale[e, r % 8, r // 8] = bits16[i, at]
            out += [words.tobytes(), scale.tobytes()]
    return np.frombuffer(b"".join(out), np.uint8)


def silu(v):
    return v / (1.0 + torch.exp(-v))


def linear(x, w, paired=False):
    """(y, bound on the kernel's error without y's own rounding) in binary64, w [n, k] as held."""
    x = x.cpu().double()
    y, size = x @ w.t(), x.abs() @ w.abs().t()
    if not paired:
        return y, SUM * size
    h = w.shape[0] // 2
    gate, up = y[:, :h], y[:, h:]
    a = silu(gate)
    # |silu'| < 1.1; exp and the quotient are good to 2^-21 of the result
    return a * up, 1.1 * SUM * size[:, :h] * up.abs() + a.abs() * SUM * size[:, h:] + 2.0 ** -20 * (a * up).abs()


def route(x, router, top, normalize):
    """(experts, weights) in binary64: largest score first, equal ones by lowest index, NaN before everything."""
    scores = x.cpu().double() @ router.cpu().double().t()
    key = torch.where(torch.isnan(scores), float("inf"), scores)
    nan = torch.isnan(scores)
    experts = torch.stack([torch.tensor(sorted(range(scores.shape[1]), key=lambda e: (not bool(nan[t, e]), -float(key[t, e]), e))[:top])
                           for t in range(scores.shape[0])]) if scores.shape[0] else torch.zeros(0, top, dtype=torch.long)
    chosen = scores.gather(1, experts)
    m = chosen[:, :1]
    over = chosen if normalize else scores
    return experts, torch.exp(chosen - m) / torch.exp(over - m).sum(1, keepdim=True)


def moe(x, router, up, down, top, normalize):
    """(y, bound without y's own rounding, experts, weights); up [e, 2 f, d] and down [e, d, f] as held."""
    experts, weights = route(x, router, top, normalize)
    y = torch.zeros(x.shape[0], down.shape[1], dtype=torch.float64)
    bound = torch.zeros_like(y)
    x = x.cpu()
    for t in range(x.shape[0]):
        for j in range(top):
            e, w = experts[t, j], weights[t, j]
            h, off = linear(x[t:t + 1], up[e], paired=True)
            h, off = w * h, w * off + (2.0 ** -17 + 2.0 ** -20) * (w * h).abs()     # held with 16 bits and more
            y[t] += (h @ down[e].t())[0]
            bound[t] += ((off + SUM * h.abs()) @ down[e].abs().t())[0]
    return y, bound, experts, weights


def check(got, want, bound):
    """got within bound of want, and its own rounding."""
    got = got.cpu()
    half = HALF_ULP[got.dtype]
    ulp = torch.finfo(got.dtype).smallest_normal * torch.finfo(got.dtype).eps
    limit = bound + half * (want.abs() + bound) + ulp
    nan = torch.isnan(want)
    assert torch.equal(torch.isnan(got), nan)
    assert bool(((got.double() - want).abs() <= limit)[~nan].all()), \
        ((got.double() - want).abs() / limit)[~nan].max()
