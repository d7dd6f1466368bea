"""Weight gradient from an 8-bit checkpoint against binary64.

The operands are exact in binary64 once the checkpoint's value is rounded to dy's type; what is left
is the binary32 sum.  A sum of `rows` products taken 16 at a time in any order is within
(rows / 16 + 24) * 2^-22 of the terms' magnitudes, where 2^-22 allows for a unit that truncates
aligned addends instead of rounding them; an accumulated or 16-bit output adds its own rounding.
"""
import numpy as np
import pytest
import torch

from train_util import HALF_ULP, TYPES, check, held64

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a CUDA device")]


def _case(seed, rows, outputs, cols, dt, group, ratio):
    from paper_2002_00104_b200 import pwlq
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.randn(rows, cols, generator=g, device="cuda") * 3
    x[:, ::7] *= 4
    dy = (torch.randn(rows, outputs, generator=g, device="cuda") * 0.1).to(dt)
    return dy, pwlq.act8_encode(x.to(dt), group=group, ratio=ratio)


def _held(saved, dt):
    """The operand's values: the checkpoint's, rounded to dy's type (bit for bit, by the decoder that
    is tested on its own)."""
    from paper_2002_00104_b200 import pwlq
    v = pwlq.act8_decode(saved, dtype=dt).double()
    exact = held64(saved)
    assert ((v - exact).abs() <= (HALF_ULP[dt] + 2.0 ** -22) * exact.abs() + 2.0 ** -25).all()
    return v


def _check(dy, saved, dw, extra_rel=0.0, base=None):
    x = _held(saved, dy.dtype)
    want = dy.double().t() @ x
    mag = dy.double().abs().t() @ x.abs()
    # two values whose 16-bit rounding is a tie may be held one ulp apart by another order of the
    # decoding operations: allowed for one value in a thousand
    slack = 2.0 ** -22 * (dy.shape[0] / 16 + 24) * mag + 2 * HALF_ULP[dy.dtype] * 1e-3 * mag
    if base is not None:
        want = want + base
        slack = slack + 2.0 ** -24 * want.abs()
    check(dw, want, slack, "dw")


SHAPES = [(1, 1, 1), (1, 4096, 300), (2, 3, 5), (16, 64, 64), (63, 128, 256), (64, 256, 128),
          (65, 257, 129), (200, 1, 513), (200, 700, 1), (333, 515, 1283), (1000, 96, 160),
          (4097, 130, 260), (2048, 1000, 512)]


@pytest.mark.parametrize("rows,outputs,cols", SHAPES)
@pytest.mark.parametrize("dtype,group", [("bf16", 128), ("fp16", 32)])
def test_sizes_and_types(rows, outputs, cols, dtype, group):
    from paper_2002_00104_b200 import pwlq
    dy, saved = _case(rows + outputs, rows, outputs, cols, TYPES[dtype], group, 0.4375)
    _check(dy, saved, pwlq.act8_weight_grad(dy, saved))
    _check(dy, saved, pwlq.act8_weight_grad(dy, saved, dtype=torch.float32))


@pytest.mark.parametrize("group", [32, 64, 128, 256])
@pytest.mark.parametrize("ratio", [0.25, 0.5, 0.75, 1.0])
def test_groups_and_ratios(group, ratio):
    from paper_2002_00104_b200 import pwlq
    dy, saved = _case(group, 300, 260, 700, torch.bfloat16, group, ratio)
    _check(dy, saved, pwlq.act8_weight_grad(dy, saved, dtype=torch.float32))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_accumulate_and_pitches(dtype):
    from paper_2002_00104_b200 import pwlq
    for off in (8, 3):
        dy, saved = _case(3, 500, 200 + 2 * off, 333, torch.bfloat16, 64, 0.5)
        part = dy[:, off:off + 200]
        store = torch.randn(200, 400, device="cuda").to(TYPES[dtype])
        keep = store.clone()
        out = store[:, off:off + 333]
        pwlq.act8_weight_grad(part, saved, out=out, accumulate=True)
        _check(part.contiguous(), saved, out.contiguous(), base=keep[:, off:off + 333].double())
        assert torch.equal(store[:, :off], keep[:, :off])
        assert torch.equal(store[:, off + 333:], keep[:, off + 333:])
        pwlq.act8_weight_grad(part, saved, out=out)
        _check(part.contiguous(), saved, out.contiguous())


def test_same_bits_again_and_on_another_stream():
    from paper_2002_00104_b200 import pwlq
    dy, saved = _case(8, 3000, 300, 400, torch.bfloat16, 128, 0.5)
    a = pwlq.act8_weight_grad(dy, saved, dtype=torch.float32)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    b = pwlq.act8_weight_grad(dy, saved, dtype=torch.float32, stream=side)
    side.synchronize()
    assert torch.equal(a, b)
    assert pwlq.device_status() == 0


def test_offsets_beyond_32_bits():
    """Rows of dy far apart: the last ones start more than 2^31 elements into it; same bits."""
    from paper_2002_00104_b200 import pwlq
    dy, saved = _case(5, 2600, 264, 272, torch.bfloat16, 64, 0.5)
    store = torch.empty(2600 << 20, dtype=torch.bfloat16, device="cuda")
    far = store.as_strided((2600, 264), (1 << 20, 1), 128)
    far.copy_(dy)
    assert torch.equal(pwlq.act8_weight_grad(far, saved), pwlq.act8_weight_grad(dy, saved))
    odd = store.as_strided((2600, 264), (1 << 20, 1), 129)
    odd.copy_(dy)
    assert torch.equal(pwlq.act8_weight_grad(odd, saved), pwlq.act8_weight_grad(dy, saved))


def test_no_rows():
    from paper_2002_00104_b200 import pwlq
    dy, saved = _case(1, 0, 20, 30, torch.bfloat16, 32, 0.5)
    out = torch.full((20, 30), 3.0, dtype=torch.bfloat16, device="cuda")
    pwlq.act8_weight_grad(dy, saved, out=out, accumulate=True)
    assert (out == 3).all()
    pwlq.act8_weight_grad(dy, saved, out=out)
    assert (out == 0).all()


def test_nan_and_infinity_reach_what_they_touch():
    from paper_2002_00104_b200 import pwlq
    dy, saved = _case(4, 100, 300, 290, torch.bfloat16, 32, 0.5)
    saved.ranges[50, 3] = float("nan")            # columns 96 ... 127
    dy[70, 299] = float("inf")
    dw = pwlq.act8_weight_grad(dy, saved, dtype=torch.float32)
    bad = torch.zeros(300, 290, dtype=torch.bool, device="cuda")
    bad[:, 96:128] = True
    bad[299] = True
    assert torch.equal(~torch.isfinite(dw), bad)


def test_refusals():
    from paper_2002_00104_b200 import pwlq
    dy, saved = _case(4, 16, 32, 48, torch.bfloat16, 32, 0.5)
    with pytest.raises(pwlq.PwlqError) as e:
        pwlq.act8_weight_grad(dy.float(), saved)
    assert e.value.status == pwlq.ERR_UNSUPPORTED
    for bad in (dy[:15], dy[0], dy.t(), dy.cpu()):
        with pytest.raises(ValueError):
            pwlq.act8_weight_grad(bad, saved)
    with pytest.raises(pwlq.PwlqError) as e:
        pwlq.act8_weight_grad(dy, saved, dtype=torch.float16)
    assert e.value.status == pwlq.ERR_INVALID_ARG
    with pytest.raises(ValueError):
        pwlq.act8_weight_grad(dy, saved, accumulate=True)
    with pytest.raises(ValueError):
        pwlq.act8_weight_grad(dy, saved, out=torch.empty(32, 47, device="cuda"))
    odd = torch.zeros(16, 33, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(pwlq.PwlqError) as e:
        pwlq.act8_weight_grad(odd, saved, workspace=torch.empty(0, dtype=torch.uint8, device="cuda"))
    assert e.value.status == pwlq.ERR_WORKSPACE
