"""The kernels that are chosen by size, at sizes derived from the device so that each of them runs."""
import pytest
import torch

from test_gpu_act8 import _check as check_checkpoint
from test_gpu_act8 import _x
from test_gpu_block_norm import KINDS, _round
from train_util import TYPES

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a CUDA device")]


def _ring_rows(cols, dtype):
    """Rows that let CTAs walk aligned rows of this width: two for each resident CTA, and a few that leave
    some CTAs a third one."""
    size = torch.empty((), dtype=dtype).element_size()
    threads = -(-cols * size // 1024) * 32                  # 32 bytes of columns each, whole warps
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    return 2 * max(1, min(16, 1024 // threads)) * sms + 37


# widths below, between and above those up to which one CTA per row takes the forward pass without checkpoints
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("cols", [1040, 1280, 2064, 4096, 8704, 12288])
@pytest.mark.parametrize("dtype,wtype", [("bf16", "bf16"), ("bf16", "fp32"), ("fp16", "fp32")])
def test_rings_of_sixteen_bit_rows(kind, cols, dtype, wtype):
    rows = _ring_rows(cols, TYPES[dtype])
    _round(rows, cols, TYPES[dtype], TYPES[wtype], kind, rows // 3, 64, 0.4375)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("cols", [520, 2056, 3584, 5128, 8192])
def test_rings_of_binary32_rows(kind, cols):
    rows = _ring_rows(cols, torch.float32)
    _round(rows, cols, torch.float32, torch.float32, kind, rows, 32, 0.5)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_gapless_checkpoints_of_many_values(dtype):
    """Above 2^25 16-bit values a thread takes three chunks of 16 to encode and four to decode; the last block
    has part of its chunks only."""
    from paper_2002_00104_b200 import pwlq
    rows, cols = 8131, 4128
    assert rows * cols > 1 << 25 and rows * cols // 16 % 768 and rows * cols // 16 % 1024
    x = _x(5, rows, cols, TYPES[dtype])
    saved = pwlq.act8_encode(x.cuda(), group=32, ratio=0.4375)
    check_checkpoint(x, 32, 0.4375, saved, pwlq.act8_decode(saved, dtype=TYPES[dtype]))


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("group,cols", [(32, 1056), (64, 1088), (128, 1152), (256, 1280)])
def test_gapless_checkpoints_of_several_blocks(dtype, group, cols):
    from paper_2002_00104_b200 import pwlq
    rows = 37                                               # blocks of 512 chunks, the last one partial
    assert rows * cols // 16 > 4 * 512 and rows * cols // 16 % 512
    x = _x(group, rows, cols, TYPES[dtype])
    saved = pwlq.act8_encode(x.cuda(), group=group, ratio=0.375)
    for out in ("fp32", dtype):
        check_checkpoint(x, group, 0.375, saved, pwlq.act8_decode(saved, dtype=TYPES[out]))


@pytest.mark.parametrize("cols,dtype", [(48, "bf16"), (512, "fp32"), (1280, "bf16"), (1283, "bf16"), (2056, "fp32"),
                                        (2047, "fp32"), (4104, "bf16"), (8704, "bf16"), (8399, "fp16")])
def test_rows_of_infinities_and_nan_stay_in_their_rows_in_every_form(cols, dtype):
    """What is not such a row has the bits that it has without them."""
    from paper_2002_00104_b200 import pwlq
    dt = TYPES[dtype]
    rows = _ring_rows(cols, dt) if cols > 512 else 1000
    g = torch.Generator(device="cuda")
    g.manual_seed(cols)
    x, f, dh, dr = (torch.randn(rows, cols, generator=g, device="cuda").to(dt) for _ in range(4))
    pre, post = (torch.rand(cols, generator=g, device="cuda").add(0.5).to(dt) for _ in range(2))
    gate = torch.rand(3, cols, generator=g, device="cuda").to(dt)
    bad = torch.zeros(rows, dtype=torch.bool, device="cuda")

    def passes():
        plain = pwlq.block_norm(x, f, pre, post, gate)[:2]
        r, h, saved = pwlq.block_norm(x, f, pre, post, gate, save=(64, 0.4375))
        grads = pwlq.block_norm_backward(saved, dh, dr)
        return [*plain, r, h, grads["dx"], grads["df"]]

    want = passes()
    for t, row, col, v in ((x, 1, 0, "inf"), (f, 3, cols - 1, "nan"), (x, rows // 2, cols // 2, "-inf"),
                           (f, rows - 1, 1, "inf"), (x, rows - 3, cols - 1, "nan")):
        t[row, col] = float(v)
        bad[row] = True
    got = passes()
    for i, (a, b) in enumerate(zip(got, want)):
        assert torch.equal(a[~bad], b[~bad])
        assert i in (0, 2) or not torch.isfinite(a[bad]).all(dim=1).any()
    dh[5, cols - 1] = float("nan")
    dr[7, 0] = float("inf")
    again = passes()
    bad[[5, 7]] = True
    for a, b in zip(again[4:], want[4:]):
        assert torch.equal(a[~bad], b[~bad])


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("cols", [512, 333])
def test_zeros_keep_their_sign_beside_other_values(dtype, cols):
    """The byte's sign is the value's sign bit, -0's too, unless the group's range is 0."""
    from paper_2002_00104_b200 import pwlq
    x = _x(1, 9, cols, TYPES[dtype])
    x[:, 1::3], x[:, 2::5], x[4, :64] = -0.0, 0.0, -0.0
    saved = pwlq.act8_encode(x.cuda(), group=64, ratio=0.4375)
    y = pwlq.act8_decode(saved, dtype=TYPES[dtype]).cpu()
    held = (saved.ranges.cpu() > 0).repeat_interleave(64, dim=1)[:, :cols]
    assert not held[4, :64].any() and held[5].all()
    negative = torch.signbit(x) & held
    assert torch.equal(saved.codes.cpu()[:, :cols] >= 128, negative)
    assert torch.equal(torch.signbit(y), negative) and (y[x == 0] == 0).all()
