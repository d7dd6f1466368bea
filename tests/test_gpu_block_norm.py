"""Norms around a gated residual block against binary64, forward and backward.

Where binary32 rounds: a sum over a row's columns is at most 32 values in a thread one after the
other and then ten levels of pairs, so it is within 48 roundings of its terms' magnitudes; the
factor rstd adds 4 (multiply-add, reciprocal square root of 2 ulp, half of the sum's); every value
then sees at most 12 more operations.  SUM, VALUE below are those counts.
"""
import numpy as np
import pytest
import torch

from train_util import (TYPES, U, act8_reference, act8_values64, backward64, check, forward64, held64,
                        on_grid)

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a CUDA device")]

SUM, VALUE = 48, 12
FACTOR = SUM / 2 + 4


def _rand(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)


def _inputs(seed, rows, cols, dtype, wtype, kind, every):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = {"x": (_rand(g, rows, cols) * 2).to(dtype), "f": None, "pre": None, "post": None, "gate": None}
    if "f" in kind:
        s["f"] = (_rand(g, rows, cols) * 0.7).to(dtype)
    if "o" in kind:
        s["post"] = (1 + 0.2 * _rand(g, cols)).to(wtype)
    if "g" in kind:
        s["gate"] = (0.5 + 0.3 * _rand(g, max(1, -(-rows // every)), cols)).to(wtype)
    if "p" in kind:
        s["pre"] = (1 + 0.2 * _rand(g, cols)).to(wtype)
    s["dh"] = (_rand(g, rows, cols) * 0.05).to(dtype) if "p" in kind else None
    s["dr"] = (_rand(g, rows, cols) * 0.05).to(dtype) if "d" in kind or "p" not in kind else None
    return s


def _d(t):
    return None if t is None else t.double()


def _check_forward(s, every, scale, eps, offset, r, h):
    w = {k: _d(s[k]) for k in ("x", "f", "pre", "post", "gate")}
    r64, h64, rr, rf = forward64(w["x"], w["f"], w["pre"], w["post"], w["gate"], every, scale, eps, offset)
    o = r64 - scale * w["x"]
    err_r = U * (VALUE * (scale * w["x"]).abs() + (VALUE + FACTOR) * o.abs())
    check(r, r64, err_r, "r")
    if h64 is not None:
        # an error of r enters h itself and, through the mean square, its factor
        rel = (err_r.square().mean(1, keepdim=True)).sqrt() * rr
        check(h, h64, err_r * rr * (w["pre"] + offset).abs() + h64.abs() * (rel + U * (VALUE + FACTOR)), "h")
    return r64, rr, rf, err_r


def _check_saved(s, saved, r64, err_r, cols, group, ratio):
    if saved.f:
        b, m, _ = act8_reference(s["f"].float().cpu().numpy(), group, ratio)
        assert np.array_equal(saved.f.codes.cpu().numpy()[:, :cols], b)
        assert not saved.f.codes[:, cols:].any()
        assert np.array_equal(saved.f.ranges.cpu().numpy(), m)
    if saved.r:
        # half a level of the piece, and what r was off in binary32
        m = saved.r.ranges.double().repeat_interleave(group, dim=1)[:, :cols]
        held = act8_values64(saved.r.codes, saved.r.ranges, cols, group, ratio)
        half = torch.where(held.abs() > ratio * m * (1 - 1e-6), (1 - ratio) * m, ratio * m) / 126
        half = torch.maximum(half, torch.where((held.abs() - ratio * m).abs() < 1e-3 * m, m / 126, 0.0))
        assert ((held - r64).abs() <= half * (1 + 1e-5) + 2 * err_r + 1e-6 * m).all()
        assert not saved.r.codes[:, cols:].any()


def _check_backward(s, every, scale, offset, saved, grads, rows_per_sum):
    w = {k: _d(s[k]) for k in ("pre", "post", "gate", "dh", "dr")}
    R = held64(saved.r) if saved.r else None
    F = held64(saved.f) if saved.f else None
    rr = saved.r_rstd.double()[:, None] if saved.r_rstd is not None else None
    rf = saved.f_rstd.double()[:, None] if saved.f_rstd is not None else None
    want, mag = backward64(R, F, rr, rf, w["dh"], w["dr"], w["pre"], w["post"], w["gate"], every, scale,
                           offset, s["f"] is not None)
    for k in ("dx", "df"):
        if k in want:
            check(grads[k], want[k], U * 2 * (SUM + 2 * VALUE) * mag[k], k)
    for k in ("dpre", "dpost", "dgate"):
        if k in want:
            check(grads[k], want[k], U * (2 * (SUM + 2 * VALUE) + rows_per_sum) * mag[k], k)
        else:
            assert grads[k] is None


# f: block output, o: norm after it, g: gate, p: norm before the next block, d: gradient on r too
KINDS = ["fogpd", "fop", "fgpd", "fpd", "pd", "p", "fog", "fo", "fg", "f"]
SHAPES = [(1, 1), (1, 4096), (2, 7), (3, 8), (17, 64), (40, 257), (33, 1000), (700, 96), (9, 2048),
          (5, 2050), (4, 4100), (6, 8192), (3, 8200), (2, 16384)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("dtype,wtype", [("bf16", "bf16"), ("fp16", "fp32"), ("fp32", "fp32")])
def test_forward_and_backward_over_sizes(rows, cols, dtype, wtype):
    _round(rows, cols, TYPES[dtype], TYPES[wtype], "fogpd", max(1, rows // 3), 64, 0.4375)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_every_combination_of_operands(kind, dtype):
    _round(37, 520, TYPES[dtype], TYPES[dtype], kind, 37, 128, 0.5)


# rows a few lanes wide, rows enough for CTAs that walk them, rows too wide for registers
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,cols", [(301, 48), (77, 512), (2400, 1280), (7, 8400),
                                       (150, 8704), (4800, 75), (3000, 1283)])
@pytest.mark.parametrize("dtype,wtype", [("bf16", "bf16"), ("bf16", "fp32"), ("fp32", "fp32")])
def test_every_combination_of_operands_in_every_form(kind, rows, cols, dtype, wtype):
    _round(rows, cols, TYPES[dtype], TYPES[wtype], kind, rows, 64, 0.4375)


@pytest.mark.parametrize("rows,cols,every", [(1, 64, 1), (5, 16, 3), (2000, 32, 2000), (1000, 96, 7),
                                             (2500, 1024, 300), (3000, 1040, 1), (2400, 2048, 2399),
                                             (300, 12288, 7), (200, 8224, 150), (4800, 333, 7),
                                             (3000, 1283, 299), (700, 4104, 150), (600, 8191, 250),
                                             (320, 9001, 20)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_gates_in_every_form(rows, cols, every, dtype):
    _round(rows, cols, TYPES[dtype], TYPES[dtype], "fogpd", every, 256, 0.5)


@pytest.mark.parametrize("group", [32, 64, 128, 256])
@pytest.mark.parametrize("every", [1, 5, 299, 1000])
def test_groups_and_gate_spans(group, every):
    _round(900, 304, torch.bfloat16, torch.float32, "fogpd", every, group, 0.375)


def _round(rows, cols, dt, wt, kind, every, group, ratio):
    from paper_2002_00104_b200 import pwlq
    s = _inputs(rows * 31 + cols, rows, cols, dt, wt, kind, every)
    scale, eps, offset = 0.75, 1e-5, 0.25
    args = dict(pre_weight=s["pre"], post_weight=s["post"], gate=s["gate"], gate_tokens=every,
                residual_scale=scale, eps=eps, weight_offset=offset)
    r, h, none = pwlq.block_norm(s["x"], s["f"], **args)
    assert none is None and (h is None) == (s["pre"] is None)
    r2, h2, saved = pwlq.block_norm(s["x"], s["f"], save=(group, ratio), **args)
    assert torch.equal(r, r2) and (h is None or torch.equal(h, h2))
    r64, rr, rf, err_r = _check_forward(s, every, scale, eps, offset, r, h)
    _check_saved(s, saved, r64, err_r, cols, group, ratio)
    if saved.f_rstd is not None:
        check(saved.f_rstd[:, None], rf, U * FACTOR * rf, "f_rstd")
    grads = pwlq.block_norm_backward(saved, s["dh"], s["dr"])
    _check_backward(s, every, scale, offset, saved, grads, -(-rows // 100) + 48)
    again = pwlq.block_norm_backward(saved, s["dh"], s["dr"])
    for k, v in grads.items():
        assert v is None or torch.equal(v, again[k])


def test_strides_in_place_and_unaligned():
    from paper_2002_00104_b200 import pwlq
    for off in (8, 3):
        g = torch.Generator(device="cuda")
        g.manual_seed(off)
        wide = _rand(g, 4, 50, 300).to(torch.bfloat16)
        x, f, dh, dr = (wide[i][:, off:off + 200] for i in range(4))
        w = (1 + 0.1 * _rand(g, 2, 200 + off)).to(torch.bfloat16)
        pre, post = w[0, off:], w[1, off:]
        gate = (_rand(g, 10, 300)).to(torch.bfloat16)[:, off:off + 200]
        args = dict(pre_weight=pre, post_weight=post, gate=gate, gate_tokens=5, residual_scale=1.5)
        want = pwlq.block_norm(x.contiguous(), f.contiguous(), save=(32, 0.5), **args)
        grads = pwlq.block_norm_backward(want[2], dh.contiguous(), dr.contiguous())
        again = pwlq.block_norm_backward(want[2], dh, dr)
        for k in grads:
            assert torch.equal(grads[k], again[k]), k
        r, h, saved = pwlq.block_norm(x, f, save=(32, 0.5), out=(x, f), **args)
        assert r.data_ptr() == x.data_ptr() and torch.equal(r, want[0]) and torch.equal(h, want[1])
        assert torch.equal(saved.r.codes, want[2].r.codes) and torch.equal(saved.f.codes, want[2].f.codes)


@pytest.mark.parametrize("kind", ["fogpd", "pd"])
@pytest.mark.parametrize("dtype,wtype", [("bf16", "bf16"), ("fp16", "fp32"), ("fp32", "fp32")])
@pytest.mark.parametrize("rows,cols", [(5000, 40), (1300, 2048), (700, 4095)])
def test_column_slices_of_wider_tensors(rows, cols, dtype, wtype, kind):
    """Every operand and result at its own offset and pitch; nothing around the results is written."""
    from paper_2002_00104_b200 import pwlq
    s = _inputs(rows + cols, rows, cols, TYPES[dtype], TYPES[wtype], kind, 130)

    def sliced(t, at, pad):
        if t is None:
            return None, None
        wide = torch.full((t.shape[0], at + t.shape[1] + pad), 7.0, dtype=t.dtype, device="cuda")
        wide[:, at:at + t.shape[1]] = t
        return wide[:, at:at + t.shape[1]], wide

    x, f, gate = sliced(s["x"], 1, 0)[0], sliced(s["f"], 3, 6)[0], sliced(s["gate"], 2, 3)[0]
    (r, wide_r), (h, wide_h) = (sliced(torch.zeros_like(s["x"]), at, pad) for at, pad in ((5, 4), (8, 1)))
    scale, eps, offset = -0.5, 1e-5, 0.25
    _, _, saved = pwlq.block_norm(x, f, gate=gate, gate_tokens=130, save=(64, 0.4375), out=(r, h),
                                  pre_weight=s["pre"], post_weight=s["post"], residual_scale=scale, eps=eps,
                                  weight_offset=offset)
    r64, _, _, err_r = _check_forward(s, 130, scale, eps, offset, r, h)
    for wide, at in ((wide_r, 5), (wide_h, 8)):
        assert (wide[:, :at] == 7).all() and (wide[:, at + cols:] == 7).all()
    _check_saved(s, saved, r64, err_r, cols, 64, 0.4375)
    grads = pwlq.block_norm_backward(saved, sliced(s["dh"], 1, 2)[0], sliced(s["dr"], 7, 0)[0])
    _check_backward(s, 130, scale, offset, saved, grads, -(-rows // 100) + 48)


def test_rows_of_zeros_infinities_and_nan_stay_in_their_rows():
    from paper_2002_00104_b200 import pwlq
    s = _inputs(77, 12, 300, torch.float32, torch.float32, "fogpd", 4)
    s["x"][1] = 0
    s["f"][1] = 0
    s["f"][3] = 0
    s["x"][5, 7] = float("inf")
    s["f"][7, 299] = float("nan")
    args = dict(pre_weight=s["pre"], post_weight=s["post"], gate=s["gate"], gate_tokens=4)
    r, h, saved = pwlq.block_norm(s["x"], s["f"], save=(64, 0.5), **args)
    grads = pwlq.block_norm_backward(saved, s["dh"], s["dr"])
    bad = torch.zeros(12, dtype=torch.bool, device="cuda")
    bad[[5, 7]] = True
    for t in (h, grads["dx"], grads["df"]):
        assert torch.equal(torch.isfinite(t).all(1), ~bad), t
    assert (r[1] == 0).all() and (h[1] == 0).all()
    # row 1: n = 0, so e = dr + dh * w / sqrt(eps)
    e = s["dr"][1].double() + s["dh"][1].double() * s["pre"].double() * 1e-6 ** -0.5
    assert torch.allclose(grads["dx"][1].double(), e, rtol=1e-5)


def test_no_rows_give_zero_sums():
    from paper_2002_00104_b200 import pwlq
    s = _inputs(1, 0, 100, torch.bfloat16, torch.float32, "fogpd", 4)
    r, h, saved = pwlq.block_norm(s["x"], s["f"], pre_weight=s["pre"], post_weight=s["post"],
                                  gate=s["gate"], save=(64, 0.5))
    grads = pwlq.block_norm_backward(saved, s["dh"], s["dr"])
    assert r.shape == (0, 100) and grads["dx"].shape == (0, 100)
    for k in ("dpre", "dpost", "dgate"):
        assert (grads[k] == 0).all()


def test_gate_rows_beyond_the_tokens_get_zero():
    from paper_2002_00104_b200 import pwlq
    s = _inputs(2, 10, 64, torch.float32, torch.float32, "fogpd", 4)
    gate = torch.ones(6, 64, device="cuda")
    _, _, saved = pwlq.block_norm(s["x"], s["f"], pre_weight=s["pre"], post_weight=s["post"], gate=gate,
                                  gate_tokens=4, save=(64, 0.5))
    d = pwlq.block_norm_backward(saved, s["dh"], s["dr"])["dgate"]
    assert (d[3:] == 0).all() and (d[:3] != 0).any(1).all()


@pytest.mark.parametrize("rows,cols", [(6, 96), (3, 2304)])
def test_gradients_against_differences(rows, cols):
    """Inputs that the checkpoints hold exactly, so that the gradient is the function's: central
    differences in binary64 of L = sum(h * dh) (plain norm) and L = sum(r * dr) (norm after the
    block and gate).  Truncation of the differences is of order step^2 * |L'''| < 1e-7 of the
    gradient's size here; the kernel's own bound is the binary32 one."""
    from paper_2002_00104_b200 import pwlq
    rng = np.random.default_rng(cols)
    grid = torch.from_numpy(on_grid(rng, rows, cols, 32, 1 / 64)).cuda()
    s = _inputs(cols, rows, cols, torch.float32, torch.float32, "fogpd", 2)
    pre, post, gate, dh, dr = (s[k] for k in ("pre", "post", "gate", "dh", "dr"))
    dirs = torch.from_numpy(rng.standard_normal((rows, cols))).cuda()

    def slope(fn, at, step=1e-4):
        def along(t):
            return fn(at + t * step * dirs[:at.shape[0], :at.shape[-1]].reshape(at.shape))
        return float((along(1) - along(-1)) / (2 * step))

    def near(grad, fn, at):
        d = dirs[:at.shape[0], :at.shape[-1]].reshape(at.shape)
        a, b = float((grad.double() * d).sum()), slope(fn, at)
        size = float((grad.double() * d).abs().sum())
        assert abs(a - b) <= 1e-5 * size + 1e-5 * abs(b), (a, b, size)

    _, _, saved = pwlq.block_norm(grid.float(), pre_weight=pre, save=(32, 0.5))
    grads = pwlq.block_norm_backward(saved, dh)
    p64, dh64 = pre.double(), dh.double()
    near(grads["dx"], lambda x: (forward64(x, None, p64, None, None, 1, 1.0, 1e-6, 0.0)[1] * dh64).sum(), grid)
    near(grads["dpre"][None], lambda w: (forward64(grid, None, w[0], None, None, 1, 1.0, 1e-6, 0.0)[1]
                                         * dh64).sum(), p64[None])
    x = s["x"]
    _, _, saved = pwlq.block_norm(x, grid.float(), post_weight=post, gate=gate, gate_tokens=2,
                                  residual_scale=0.5, save=(32, 0.5))
    grads = pwlq.block_norm_backward(saved, dr=dr)
    o64, g64, dr64, x64 = post.double(), gate.double(), dr.double(), x.double()

    def loss(f, o, g):
        return (forward64(x64, f, None, o, g, 2, 0.5, 1e-6, 0.0)[0] * dr64).sum()

    near(grads["df"], lambda f: loss(f, o64, g64), grid)
    near(grads["dpost"][None], lambda o: loss(grid, o[0], g64), o64[None])
    near(grads["dgate"], lambda g: loss(grid, o64, g), g64)
    assert torch.equal(grads["dx"], 0.5 * dr)


def test_another_stream():
    from paper_2002_00104_b200 import pwlq
    s = _inputs(5, 64, 512, torch.bfloat16, torch.bfloat16, "fogpd", 8)
    args = dict(pre_weight=s["pre"], post_weight=s["post"], gate=s["gate"], gate_tokens=8, save=(64, 0.5))
    want = pwlq.block_norm(s["x"], s["f"], **args)
    want_g = pwlq.block_norm_backward(want[2], s["dh"], s["dr"])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    r, h, saved = pwlq.block_norm(s["x"], s["f"], stream=side, **args)
    grads = pwlq.block_norm_backward(saved, s["dh"], s["dr"], stream=side)
    side.synchronize()
    assert torch.equal(r, want[0]) and torch.equal(h, want[1])
    for k in grads:
        assert torch.equal(grads[k], want_g[k])


def test_refusals():
    from paper_2002_00104_b200 import pwlq
    x = torch.zeros(4, 64, device="cuda")
    w = torch.ones(64, device="cuda")
    gate = torch.ones(2, 64, device="cuda")

    def refused(exc, status=None, **kw):
        base = dict(x=x, f=x, pre_weight=w)
        base.update(kw)
        with pytest.raises(exc) as e:
            pwlq.block_norm(base.pop("x"), base.pop("f"), **base)
        assert status is None or e.value.status == status

    refused(pwlq.PwlqError, pwlq.ERR_INVALID_ARG, gate=gate, gate_tokens=1)       # 2 gates, 4 rows
    refused(pwlq.PwlqError, pwlq.ERR_INVALID_ARG, f=None, gate=gate, gate_tokens=2)
    refused(pwlq.PwlqError, pwlq.ERR_INVALID_ARG, save=(48, 0.5))
    refused(pwlq.PwlqError, pwlq.ERR_INVALID_ARG, save=(64, 2.0))
    wide = torch.zeros(1, pwlq.BLOCK_NORM_MAX_COLS + 1, device="cuda")
    refused(pwlq.PwlqError, pwlq.ERR_UNSUPPORTED, x=wide, f=None, pre_weight=wide[0])
    refused(ValueError, f=x.bfloat16())
    refused(ValueError, f=x[:3])
    refused(ValueError, pre_weight=w[:63])
    refused(ValueError, pre_weight=w.bfloat16(), post_weight=w)
    refused(ValueError, pre_weight=w.half())
    refused(ValueError, x=x.t().contiguous().t())
    _, _, saved = pwlq.block_norm(x, x, pre_weight=w, post_weight=w, save=(64, 0.5))
    for bad in (dict(dh=None, dr=x), dict(dh=x[:3]), dict(dh=x.bfloat16()), dict()):
        with pytest.raises(ValueError):
            pwlq.block_norm_backward(saved, **bad)
    small = torch.empty(256, dtype=torch.uint8, device="cuda")
    with pytest.raises(pwlq.PwlqError) as e:
        pwlq.block_norm_backward(saved, x, workspace=small)
    assert e.value.status == pwlq.ERR_WORKSPACE


@pytest.mark.parametrize("cols", [512, 1024, 4001])
def test_offsets_beyond_32_bits(cols):
    """Rows far apart: the last ones start more than 2^31 elements into their tensors.  The results are
    those of contiguous rows."""
    from paper_2002_00104_b200 import pwlq
    rows, pitch = 2600, 1 << 20
    s = _inputs(cols, rows, cols, torch.bfloat16, torch.bfloat16, "fogpd", 700)
    store = torch.empty(rows * pitch, dtype=torch.bfloat16, device="cuda")
    far = [store.as_strided((rows, cols), (pitch, 1), 16384 * i + cols % 2) for i in range(6)]
    for to, k in zip(far, ("x", "f", "dh", "dr")):
        to.copy_(s[k])
    args = dict(pre_weight=s["pre"], post_weight=s["post"], gate=s["gate"], gate_tokens=700)
    near = [torch.empty(rows, cols + 16, dtype=torch.bfloat16, device="cuda")[:, :cols] for _ in range(6)]
    for to, k in zip(near, ("x", "f", "dh", "dr")):
        to.copy_(s[k])
    for save in (None, (64, 0.5)):
        r, h, saved = pwlq.block_norm(far[0], far[1], save=save, out=(far[4], far[5]), **args)
        r2, h2, saved2 = pwlq.block_norm(near[0], near[1], save=save, out=(near[4], near[5]), **args)
        assert torch.equal(r, r2) and torch.equal(h, h2)
    assert torch.equal(saved.r.codes, saved2.r.codes) and torch.equal(saved.f.codes, saved2.f.codes)
    got = pwlq.block_norm_backward(saved, far[2], far[3])
    want = pwlq.block_norm_backward(saved2, near[2], near[3])
    for k in want:
        assert torch.equal(got[k], want[k]), k
