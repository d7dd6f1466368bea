"""4-bit weights: format, byte for byte, and the product of a few tokens with them."""
import numpy as np
import pytest
import torch

import w4_util as U
from w4_util import TYPES

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a CUDA device")]


def _w(seed, *shape, dtype=torch.float32, scale=0.05):
    rng = np.random.default_rng(seed)
    return torch.from_numpy((rng.standard_t(4, shape) * scale).astype(np.float32)).to(dtype)


def _same(got, want):
    got = got.cpu()
    want = want.to(got.dtype)
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(want))


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("rows,cols,group,ratio,paired", [
    (1, 1, 32, 0.5, False), (2, 1, 64, 0.25, True), (16, 128, 128, 0.421875, False), (17, 129, 64, 0.4375, False),
    (5, 31, 256, 1.0, False), (33, 700, 256, 1 / 64, False), (18, 333, 32, 0.5, True), (34, 257, 64, 0.375, True),
    (64, 385, 128, 63 / 64, True), (100, 96, 32, 0.3125, False), (40, 512, 32, 1.0, False)])
def test_bytes_and_values(dtype, rows, cols, group, ratio, paired):
    from paper_2002_00104_b200 import pwlq
    w = _w(rows * 1009 + cols, rows, cols, dtype=TYPES[dtype])
    packed = pwlq.w4_encode(w.cuda(), group=group, ratio=ratio, paired=paired)
    s, c = U.codes(w.float(), group, ratio)
    assert np.array_equal(packed.memory.cpu().numpy(), U.layout(s, c, group, paired))
    for out in ("fp32", dtype):
        _same(pwlq.w4_decode(packed, dtype=TYPES[out]), U.values(s, c, group, ratio))


def test_values_on_the_bounds_between_levels():
    """Every bound and its two neighbours in binary32; the group's first value sets the scale."""
    from paper_2002_00104_b200 import pwlq
    for b in (1, 20, 27, 32, 63, 64):
        s = np.float32(2.0 ** -7 * 1.40625)              # a bfloat16
        n = [k * b for k in (0.5, 1, 1.5, 2, 2.5, 3)] + [3 * b + k * (64 - b) for k in (0, 0.5, 1, 1.5, 2, 2.5, 3)]
        v = np.array([np.float32(k) * s for k in n], np.float32)
        v = np.concatenate([v, np.nextafter(v, np.float32(0)), np.nextafter(v, np.float32(9)).clip(max=192 * s)])
        w = np.zeros((2, 64), np.float32)
        w[0, 1:1 + v.size], w[1, 1:1 + v.size] = v, -v
        w[:, 0] = 192 * s
        w = torch.from_numpy(w)
        packed = pwlq.w4_encode(w.cuda(), group=64, ratio=b / 64)
        assert np.array_equal(packed.memory.cpu().numpy(), U.layout(*U.codes(w, 64, b / 64), 64, False))
        _same(pwlq.w4_decode(packed), U.held(w, 64, b / 64))


def test_groups_of_zeros_tiny_and_large_values_infinities_and_nan():
    from paper_2002_00104_b200 import pwlq
    w = _w(3, 12, 200)
    w[0, :64] = 0.0
    w[1, 5] = float("inf")
    w[2, 70] = float("nan")
    w[3, 64:128] *= 2.0 ** -130
    w[4] = 2.0 ** -101
    w[5, :64] = 0.0
    w[5, 3] = 2.0 ** -100
    w[6] *= 2.0 ** 120
    w[7, 199] = -float("inf")
    w[8, :] = -0.0
    packed = pwlq.w4_encode(w.cuda(), group=64, ratio=0.4375)
    want = U.held(w, 64, 0.4375)
    assert torch.isnan(want[1, :64]).all() and not torch.isnan(want[1, 64:]).any()
    _same(pwlq.w4_decode(packed), want)


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("offset,pad", [(0, 8), (1, 0), (3, 5), (8, 24)])
def test_slices_and_outputs_off_their_alignment(dtype, offset, pad):
    from paper_2002_00104_b200 import pwlq
    dt = TYPES[dtype]
    wide = _w(5, 3, 21, offset + 333 + pad, dtype=dt).cuda()
    w = wide[:, :20, offset:offset + 333]
    packed = pwlq.w4_encode(w, group=64, ratio=0.375)
    y = torch.full_like(wide, 7.0)
    pwlq.w4_decode(packed, out=y[:, :20, offset:offset + 333])
    _same(y[:, :20, offset:offset + 333], U.held(w, 64, 0.375))
    assert (y[..., :offset] == 7).all() and (y[..., offset + 333:] == 7).all() and (y[:, 20:] == 7).all()
    assert torch.equal(pwlq.w4_encode(w.contiguous(), group=64, ratio=0.375).memory, packed.memory)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,cols,paired", [(994, 1000, True), (1001, 777, False), (1000, 768, True)])
def test_many_matrices_at_once(dtype, rows, cols, paired):
    """Enough of them that a CTA goes through several tiles, and not whole numbers of these."""
    from paper_2002_00104_b200 import pwlq
    w = (torch.randn(40, rows, cols, generator=torch.Generator("cuda").manual_seed(rows), device="cuda") * 0.05).to(TYPES[dtype])
    packed = pwlq.w4_encode(w, group=256, ratio=0.375, paired=paired)
    each = [pwlq.w4_encode(v, group=256, ratio=0.375, paired=paired).memory for v in w]
    assert torch.equal(packed.memory, torch.cat(each))
    _same(pwlq.w4_decode(packed)[39], U.held(w[39], 256, 0.375))


def test_memory_that_is_written_again():
    from paper_2002_00104_b200 import pwlq
    a, b = _w(1, 40, 300).cuda(), _w(2, 40, 300).cuda()
    packed = pwlq.w4_encode(a, group=32, ratio=0.25)
    packed.memory.fill_(255)
    assert pwlq.w4_encode(b, out=packed) is packed
    fresh = pwlq.w4_encode(b, group=32, ratio=0.25)
    assert torch.equal(packed.memory, fresh.memory)
    again = pwlq.W4(fresh.memory.clone(), fresh.shape, fresh.group, fresh.ratio, fresh.paired)
    assert torch.equal(pwlq.w4_decode(again), pwlq.w4_decode(fresh))


SHAPES = [(1, 1, 1, 32), (1, 16, 128, 128), (1, 17, 127, 64), (2, 4096, 64, 32), (3, 100, 1000, 256), (5, 333, 1285, 32),
          (7, 16, 8192, 128), (8, 500, 520, 64), (9, 48, 640, 128), (13, 33, 4096, 64), (16, 130, 1025, 128),
          (17, 64, 256, 32), (31, 70, 900, 64), (33, 96, 384, 128), (64, 200, 2048, 64), (100, 40, 515, 256), (1, 4112, 8200, 128),
          (4, 4097, 8192, 64), (5, 8000, 1030, 32), (12, 6001, 1601, 64), (32, 5000, 1700, 64), (33, 8193, 200, 128),
          (64, 8200, 520, 32), (65, 100, 300, 64), (130, 256, 4096, 128)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("tokens,rows,cols,group", SHAPES)
def test_products_of_whole_numbers_are_exact(dtype, tokens, rows, cols, group):
    """Scales of one power of two and whole activations: every sum is a whole number below 2^24 times that power,
    whatever the order; what is delivered is its rounding."""
    from paper_2002_00104_b200 import pwlq
    dt = TYPES[dtype]
    rng = np.random.default_rng(tokens * rows + cols)
    b = 24
    levels = np.array([0, 24, 48, 72, 112, 152, 192], np.float32)
    n = levels[rng.integers(0, 7, (rows, cols))] * rng.choice([-1, 1], (rows, cols))
    n[:, ::group] = 192                                  # every group's scale
    w = torch.from_numpy((n * 2.0 ** -9).astype(np.float32))
    x = torch.from_numpy(rng.integers(-3, 4, (tokens, cols)).astype(np.float32)).to(dt)
    want = x.double() @ torch.from_numpy(n).double().t() * 2.0 ** -9
    packed = pwlq.w4_encode(w.cuda(), group=group, ratio=b / 64)
    _same(pwlq.w4_linear(x.cuda(), packed), want)


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("paired", [False, True])
@pytest.mark.parametrize("tokens,rows,cols,group", [(1, 2, 1, 64), (1, 1000, 2048, 64), (6, 36, 777, 32), (8, 8, 9000, 128),
                                                    (12, 130, 384, 256), (40, 34, 1029, 64), (64, 256, 512, 128), (70, 66, 777, 64)])
def test_products(dtype, paired, tokens, rows, cols, group):
    from paper_2002_00104_b200 import pwlq
    dt = TYPES[dtype]
    w, x = _w(rows + cols, rows, cols, dtype=dt), _w(tokens, tokens, cols, dtype=dt, scale=1.0)
    packed = pwlq.w4_encode(w.cuda(), group=group, ratio=0.421875, paired=paired)
    y = pwlq.w4_linear(x.cuda(), packed)
    U.check(y, *U.linear(x, U.held(w, group, 0.421875), paired))
    assert torch.equal(y, pwlq.w4_linear(x.cuda(), packed))          # the same bits every time


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("tokens", [1, 3, 20])
def test_rows_off_their_alignment_and_what_lies_around_them(dtype, tokens):
    from paper_2002_00104_b200 import pwlq
    dt = TYPES[dtype]
    for cols, off in ((256, 1), (256, 8), (300, 5), (129, 0)):
        wide = torch.full((tokens, off + cols + 3), float("nan"), dtype=dt)
        wide[:, off:off + cols] = _w(cols, tokens, cols, dtype=dt, scale=1.0)
        x = wide.cuda()[:, off:off + cols]
        w = _w(9, 50, cols, dtype=dt)
        packed = pwlq.w4_encode(w.cuda(), group=64, ratio=0.5)
        out = torch.full((tokens, 61), 7.0, dtype=dt, device="cuda")
        y = pwlq.w4_linear(x, packed, out=out[:, 5:55])
        U.check(y, *U.linear(wide[:, off:off + cols], U.held(w, 64, 0.5)))
        assert torch.equal(y, pwlq.w4_linear(x.contiguous(), packed))
        assert (out[:, :5] == 7).all() and (out[:, 55:] == 7).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("cols", [256, 300])
def test_infinities_and_nan_stay_in_their_rows(dtype, cols):
    from paper_2002_00104_b200 import pwlq
    dt = TYPES[dtype]
    w, x = _w(4, 48, cols), _w(5, 6, cols, dtype=dt, scale=1.0)
    w[3, 40] = float("nan")                              # a row's outputs
    w[2, 33], w[2, 7] = 0.0, 1.0
    packed = pwlq.w4_encode(w.cuda(), group=64, ratio=0.5)
    clean = pwlq.w4_linear(x.cuda(), packed)
    x[1, 7], x[4, 100] = float("inf"), float("nan")
    y = pwlq.w4_linear(x.cuda(), packed)
    assert torch.isnan(y[:, 3]).all() and torch.isnan(clean[:, 3]).all()
    keep = [t for t in range(6) if t not in (1, 4)]
    assert torch.equal(torch.nan_to_num(y[keep]), torch.nan_to_num(clean[keep]))
    assert torch.isnan(y[4]).all()
    held = U.held(w, 64, 0.5)
    want = x[1:2].double() @ held.t()                    # +-infinity, or NaN where the weight is held as 0
    assert torch.equal(torch.isnan(y[1].cpu()), torch.isnan(want[0]))
    assert torch.equal(y[1].cpu().double()[~torch.isnan(want[0])], want[0][~torch.isnan(want[0])])


def test_largest_and_smallest_activations():
    """Sums of large values that cancel stay finite; binary32 values keep all their bits."""
    from paper_2002_00104_b200 import pwlq
    w = torch.zeros(16, 128)
    w[:, 0] = 192.0
    w[0, 1], w[1, 2], w[2, 3] = 192.0, 64.0, -128.0
    packed = pwlq.w4_encode(w.cuda(), group=128, ratio=1.0)
    x = torch.zeros(4, 128)
    x[0, 0], x[0, 1] = 2.0 ** 100, -2.0 ** 100
    x[1, 2] = float(np.nextafter(np.float32(1), np.float32(2)))
    x[2, 3] = 1.0 + 2.0 ** -23 + 2.0 ** -12
    x[3, 0] = 2.0 ** -100
    y = pwlq.w4_linear(x.cuda(), packed).cpu()
    assert torch.equal(y.double(), (x.double() @ U.held(w, 128, 1.0).t()).float().double())


@pytest.mark.parametrize("dtype,cols", [("fp32", 256), ("bf16", 129), ("bf16", 300), ("fp16", 300)])
def test_workspaces(dtype, cols):
    from paper_2002_00104_b200 import pwlq
    dt = TYPES[dtype]
    rows = 16 * 2100
    w, x = _w(1, rows, cols), _w(2, 5, cols, dtype=dt, scale=1.0)
    x[2, 7], x[4, cols - 1] = float("inf"), float("nan")
    packed, x = pwlq.w4_encode(w.cuda()), x.cuda()
    need = pwlq.w4_linear_workspace_bytes(5, rows, cols, dt)
    assert need > 0
    few = pwlq.w4_linear(x, pwlq.w4_encode(w[:4096].cuda()))         # without a copy
    assert pwlq.w4_linear_workspace_bytes(5, 4096, cols, dt) == 0
    assert torch.equal(torch.nan_to_num(pwlq.w4_linear(x, packed)[:, :4096], 7.0), torch.nan_to_num(few, 7.0))
    x = x.nan_to_num(1.0, 1.0)
    workspace = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    assert torch.equal(pwlq.w4_linear(x, packed, workspace=workspace), pwlq.w4_linear(x, packed))
    with pytest.raises(pwlq.PwlqError) as e:
        pwlq.w4_linear(x, packed, workspace=workspace[:-1])
    assert e.value.status == pwlq.ERR_WORKSPACE
    with pytest.raises(ValueError):
        pwlq.w4_linear(x, packed, workspace=workspace.cpu())


def test_no_tokens():
    from paper_2002_00104_b200 import pwlq
    packed = pwlq.w4_encode(_w(1, 20, 100).cuda(), paired=True)
    assert pwlq.w4_linear(torch.zeros(0, 100, device="cuda"), packed).shape == (0, 10)


def test_refusals():
    from paper_2002_00104_b200 import pwlq
    w = _w(1, 32, 256).cuda()
    packed, x = pwlq.w4_encode(w), torch.zeros(4, 256, device="cuda")
    several = pwlq.w4_encode(w.view(2, 16, 256))
    out = torch.zeros(4, 32, device="cuda")
    for bad in (lambda: pwlq.w4_encode(w.half().double()), lambda: pwlq.w4_encode(w.t()), lambda: pwlq.w4_encode(w[0].expand(4, 256)),
                lambda: pwlq.w4_encode(w, out=several), lambda: pwlq.w4_encode(w.cpu()),
                lambda: pwlq.w4_decode(packed, dtype=torch.float64), lambda: pwlq.w4_decode(packed, out=torch.zeros(32, 255, device="cuda")),
                lambda: pwlq.w4_decode(several, out=torch.zeros(16, 256, device="cuda").expand(2, 16, 256)),
                lambda: pwlq.w4_linear(x[:, :255], packed), lambda: pwlq.w4_linear(x.double(), packed),
                lambda: pwlq.w4_linear(x.t(), packed), lambda: pwlq.w4_linear(x[0], packed),
                lambda: pwlq.w4_linear(x, packed, out=out.half()), lambda: pwlq.w4_linear(x, packed, out=out[:3]),
                lambda: pwlq.w4_linear(x, pwlq.W4(packed.memory.cpu(), packed.shape)),
                lambda: pwlq.w4_linear(x.requires_grad_(), packed)):
        with pytest.raises(ValueError):
            bad()
    x = x.detach()
    with torch.no_grad():
        pwlq.w4_linear(x.requires_grad_(), packed)
    x = x.detach()
    square = pwlq.w4_encode(_w(2, 256, 256).cuda())
    shifted = torch.zeros(square.memory.numel() + 8, dtype=torch.uint8, device="cuda")[8:]
    for bad in (lambda: pwlq.w4_linear(x, several), lambda: pwlq.w4_linear(x, square, out=x),
                lambda: pwlq.w4_linear(x, pwlq.W4(shifted, square.shape))):
        with pytest.raises(pwlq.PwlqError) as e:
            bad()
        assert e.value.status == pwlq.ERR_INVALID_ARG


def test_rows_far_apart():
    """Token rows more than 2^31 bytes from each other, in and out."""
    from paper_2002_00104_b200 import pwlq
    w = _w(6, 40, 512, dtype=torch.bfloat16)
    packed = pwlq.w4_encode(w.cuda(), group=64, ratio=0.5)
    far = torch.empty(3, 1 << 30, dtype=torch.bfloat16, device="cuda")
    x = _w(7, 3, 512, dtype=torch.bfloat16, scale=1.0).cuda()
    far[:, :512] = x
    y = pwlq.w4_linear(far[:, :512], packed, out=far[:, 1024:1064])
    assert torch.equal(y, pwlq.w4_linear(x, packed))


@pytest.mark.parametrize("cols", [1023, 1024])
def test_very_many_tokens(cols):
    """More than a grid's second axis holds, of rows that are copied first and of others."""
    from paper_2002_00104_b200 import pwlq
    packed = pwlq.w4_encode(_w(8, 8192, cols, dtype=torch.bfloat16).cuda(), group=64)
    x = torch.randn(66001, cols, generator=torch.Generator("cuda").manual_seed(1), device="cuda").bfloat16()
    y = pwlq.w4_linear(x, packed)
    for at in (0, 65520, 65536, 65990):
        assert torch.equal(y[at:at + 11], pwlq.w4_linear(x[at:at + 11], packed))


def test_best_ratio_of_a_weight_matrix():
    from paper_2002_00104_b200 import pwlq, training
    w = _w(8, 64, 1024).cuda()
    best = training.best_ratio(w, group=128, candidates=64, bits=3)
    error = {}
    for ratio in (0.25, best, 0.75):
        error[ratio] = float((pwlq.w4_decode(pwlq.w4_encode(w, ratio=ratio)) - w).square().sum())
    assert error[best] <= min(error.values()) * 1.01     # the search takes ranges in 32 bits, the format in 8
