"""8-bit checkpoints against the format's definition, byte for byte, and their refusals."""
import numpy as np
import pytest
import torch

from train_util import TYPES, act8_reference

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a CUDA device")]


def _x(seed, rows, cols, dtype, scale=1.0):
    rng = np.random.default_rng(seed)
    v = (rng.standard_t(4, (rows, cols)) * scale).astype(np.float32)
    return torch.from_numpy(v).to(dtype)


def _check(x, group, ratio, saved, y):
    want_b, want_m, want_y = act8_reference(x.float().cpu().numpy(), group, ratio)
    cols = x.shape[1]
    codes = saved.codes.cpu().numpy()
    assert np.array_equal(saved.ranges.cpu().numpy().view(np.int32), want_m.view(np.int32))
    assert np.array_equal(codes[:, :cols], want_b)
    assert not codes[:, cols:].any()
    want = torch.from_numpy(want_y).to(y.dtype)
    got = y.cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(want))


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("rows,cols,group,ratio", [
    (1, 1, 32, 0.5), (1, 4096, 128, 0.4375), (3, 15, 32, 0.25), (2, 16, 64, 0.5), (5, 17, 32, 1.0),
    (7, 333, 128, 0.375), (33, 255, 256, 0.3), (64, 1000, 64, 0.5), (9, 4095, 128, 0.4375),
    (3, 4097, 256, 0.5), (2, 12289, 128, 0.625), (300, 40, 32, 2.0 ** -20)])
def test_bytes_ranges_and_values(dtype, rows, cols, group, ratio):
    from paper_2002_00104_b200 import pwlq
    x = _x(rows * 7919 + cols, rows, cols, TYPES[dtype])
    saved = pwlq.act8_encode(x.cuda(), group=group, ratio=ratio)
    for out in ("fp32", dtype):
        _check(x, group, ratio, saved, pwlq.act8_decode(saved, dtype=TYPES[out]))


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("offset,pad", [(0, 8), (1, 0), (3, 5), (8, 24)])
def test_column_slices_and_outputs_off_their_alignment(dtype, offset, pad):
    from paper_2002_00104_b200 import pwlq
    dt = TYPES[dtype]
    wide = _x(5, 21, offset + 777 + pad, dt).cuda()
    x = wide[:, offset:offset + 777]
    saved = pwlq.act8_encode(x, group=64, ratio=0.375)
    y = torch.full((21, offset + 777 + pad), 7.0, dtype=dt, device="cuda")
    pwlq.act8_decode(saved, out=y[:, offset:offset + 777])
    _check(x.cpu(), 64, 0.375, saved, y[:, offset:offset + 777])
    assert (y[:, :offset] == 7).all() and (y[:, offset + 777:] == 7).all()


def test_groups_of_zeros_tiny_values_infinities_and_nan():
    from paper_2002_00104_b200 import pwlq
    x = _x(11, 12, 200, torch.float32)
    x[0, :64] = 0.0
    x[1, 64:128] = -0.0
    x[2, :64] = 2.0 ** -101                       # below the smallest range that is kept
    x[3, :64] = 0.0
    x[3, 5] = -2.0 ** -100                        # the smallest one
    x[4, 70] = float("inf")
    x[5, 199] = float("-inf")
    x[6, 3] = float("nan")
    x[7, :64] = 2.0 ** -140                       # subnormal
    x[8, :64] *= 1e37
    saved = pwlq.act8_encode(x.cuda(), group=64, ratio=0.5)
    y = pwlq.act8_decode(saved)
    _check(x, 64, 0.5, saved, y)
    y = y.cpu()
    assert (y[0, :64] == 0).all() and (y[2, :64] == 0).all() and y[3, 5] == -2.0 ** -100
    assert torch.isnan(y[4, 64:128]).all() and not torch.isnan(y[4, :64]).any()
    assert torch.isnan(y[5, 192:]).all() and torch.isnan(y[6, :64]).all()


def test_no_rows_reuse_of_a_checkpoint_and_another_stream():
    from paper_2002_00104_b200 import pwlq
    empty = pwlq.act8_encode(torch.empty(0, 100, device="cuda"))
    assert empty.codes.shape == (0, 112) and pwlq.act8_decode(empty).shape == (0, 100)
    x = _x(3, 50, 300, torch.bfloat16)
    side = torch.cuda.Stream()
    xd = x.cuda()
    out = pwlq.act8_empty(50, 300, 128, 0.5, "cuda")
    out.codes.fill_(255)
    side.wait_stream(torch.cuda.current_stream())
    saved = pwlq.act8_encode(xd, out=out, stream=side)
    y = pwlq.act8_decode(saved, dtype=torch.bfloat16, stream=side)
    side.synchronize()
    assert saved is out
    again = pwlq.Act8(saved.codes, saved.ranges, 300, 128, 0.5)       # the same, from its two tensors
    assert torch.equal(pwlq.act8_decode(again, dtype=torch.bfloat16), y)
    want_b, _, want_y = act8_reference(x.float().numpy(), 128, 0.5)
    assert np.array_equal(saved.codes.cpu().numpy()[:, :300], want_b)
    assert torch.equal(y.cpu(), torch.from_numpy(want_y).to(torch.bfloat16))


def test_offsets_beyond_32_bits():
    """Rows far apart: the last row starts more than 2^31 elements into x."""
    from paper_2002_00104_b200 import pwlq
    rows, pitch, cols = 5, (1 << 29) + 8, 100
    store = torch.empty(rows * pitch, dtype=torch.bfloat16, device="cuda")
    x = store.as_strided((rows, cols), (pitch, 1))
    x.copy_(_x(9, rows, cols, torch.bfloat16))
    saved = pwlq.act8_encode(x, group=32, ratio=0.5)
    back = store.as_strided((rows, cols), (pitch, 1), 128)
    pwlq.act8_decode(saved, out=back)
    _check(x.cpu(), 32, 0.5, saved, back.contiguous())


def test_held_values_are_those_of_the_seven_bit_quantizer(oracle):
    """Against the oracle's quantizer, one row per group: the same level and region, except where the
    value lies half way between two levels within the rounding of the constants (there one level)."""
    from paper_2002_00104_b200 import pwlq
    x = _x(21, 200, 1024, torch.float32)
    saved = pwlq.act8_encode(x.cuda(), group=64, ratio=0.4375)
    y = pwlq.act8_decode(saved).cpu().numpy().reshape(-1, 64)
    m = saved.ranges.cpu().numpy().reshape(-1)
    p = m * np.float32(0.4375)
    codes, mask, fake = oracle.quantize(x.numpy().reshape(-1, 64), 7, m, p, layout=0)
    off = np.abs(y - fake.reshape(-1, 64)) / m[:, None]
    assert (off <= 1.01 * 0.5625 / 63).all()
    assert (off > 4 * 2.0 ** -24).mean() < 1e-4
    region = np.unpackbits(mask, bitorder="little")[:x.numel()].reshape(200, -1)
    assert np.array_equal(saved.codes.cpu().numpy() >> 6 & 1, region)


def test_refusals():
    from paper_2002_00104_b200 import pwlq
    x = torch.zeros(4, 64, device="cuda")
    for bad in (dict(group=48), dict(ratio=0.0), dict(ratio=1.5), dict(ratio=float("nan"))):
        with pytest.raises(pwlq.PwlqError) as e:
            pwlq.act8_encode(x, **bad)
        assert e.value.status == pwlq.ERR_INVALID_ARG
    for bad in (x.cpu(), x.double(), x[0], x.t(), x[:1].expand(4, 64)):
        with pytest.raises(ValueError):
            pwlq.act8_encode(bad)
    with pytest.raises(ValueError):
        pwlq.act8_encode(x, out=pwlq.act8_empty(4, 128, device="cuda"))
    saved = pwlq.act8_encode(x)
    with pytest.raises(ValueError):
        pwlq.act8_decode(pwlq.Act8(saved.codes[:, :60], saved.ranges, 64, 128, 0.5))
    with pytest.raises(ValueError):
        pwlq.act8_decode(pwlq.Act8(saved.codes, saved.ranges[:3], 64, 128, 0.5))
    with pytest.raises(ValueError):
        pwlq.act8_decode(saved, out=torch.empty(4, 63, device="cuda"))
