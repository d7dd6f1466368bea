"""Weight gradients of more tiles than there are pairs of CTAs (several units of work per pair, whole tiles
and pieces together), and their whole error.

Against binary64 at the checkpoint's own values.  x_hat is rounded to dy's type (within half an ulp of it),
the products are exact, and a sum of `rows` of them taken 16 at a time in any order is within
(rows / 16 + 24) * 2^-22 of the terms' magnitudes.
"""
import pytest
import torch

from train_util import HALF_ULP, SUBNORMAL, TYPES, check, held64

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a CUDA device")]


def _case(rows, outputs, cols, dt, group=128, ratio=0.4375):
    from paper_2002_00104_b200 import pwlq
    g = torch.Generator(device="cuda")
    g.manual_seed(rows + outputs + cols)
    x = torch.randn(rows, cols, generator=g, device="cuda") * 3
    dy = (torch.randn(rows, outputs, generator=g, device="cuda") * 0.1).to(dt)
    return dy, pwlq.act8_encode(x.to(dt), group=group, ratio=ratio)


def _check(dy, saved, dw, base=None):
    x, d = held64(saved), dy.double()
    rows, dt = dy.shape[0], dy.dtype
    want, mag = d.t() @ x, d.abs().t() @ x.abs()
    # the decoder's own binary32 operations, then the rounding to dy's type
    slack = (2.0 ** -22 * (rows / 16 + 24 + 1) + HALF_ULP[dt]) * mag
    slack += SUBNORMAL[dt] * d.abs().sum(0)[:, None]
    if base is not None:
        want = want + base
        slack = slack + 2.0 ** -24 * want.abs()
    check(dw, want, slack, "dw")


def _tiles(outputs, cols):
    return -(-outputs // 256) * -(-cols // 256)


def _pairs():
    return torch.cuda.get_device_properties(0).multi_processor_count // 2


# (rows, outputs, cols): steps of 64 rows; 24 of them and more allow a last round of tiles to be cut
UNCUT = [(200, 4096, 2560), (70, 5000, 4100), (1, 4097, 4097)]
CUT = [(2048, 3000, 2570), (1700, 4096, 2560), (4097, 2563, 2050), (1536, 300, 19001)]


@pytest.mark.parametrize("rows,outputs,cols", UNCUT + CUT)
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_several_units_per_pair(rows, outputs, cols, dtype):
    from paper_2002_00104_b200 import pwlq
    dt = TYPES[dtype]
    assert _tiles(outputs, cols) > _pairs()
    if (rows, outputs, cols) in UNCUT[:2]:
        assert _tiles(outputs, cols) > 2 * _pairs()
    dy, saved = _case(rows, outputs, cols, dt)
    a = pwlq.act8_weight_grad(dy, saved, dtype=torch.float32)
    _check(dy, saved, a)
    assert torch.equal(a, pwlq.act8_weight_grad(dy, saved, dtype=torch.float32))
    b = pwlq.act8_weight_grad(dy, saved)
    _check(dy, saved, b)
    assert torch.equal(b, a.to(dt))
    for kind in (torch.float32, dt):
        store = torch.randn(outputs, cols + 5, device="cuda").to(kind)
        keep, out = store.clone(), store[:, 2:cols + 2]
        pwlq.act8_weight_grad(dy, saved, out=out, accumulate=True)
        _check(dy, saved, out, base=keep[:, 2:cols + 2].double())
        assert torch.equal(store[:, :2], keep[:, :2]) and torch.equal(store[:, cols + 2:], keep[:, cols + 2:])
    assert pwlq.device_status() == 0


@pytest.mark.parametrize("tiles", [1, 36, 37, 38, 73, 74, 75, 111, 148, 149, 185, 222])
def test_every_kind_of_last_round(tiles):
    """One row of tiles, 24 steps: from uncut single rounds to whole rounds with one tile or most of a round
    left over."""
    from paper_2002_00104_b200 import pwlq
    dy, saved = _case(24 * 64, 130, 256 * tiles - 120, torch.bfloat16, group=64)
    _check(dy, saved, pwlq.act8_weight_grad(dy, saved, dtype=torch.float32))


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_the_operand_s_rounding_is_all_that_is_lost(dtype):
    """A sum of many terms: the relative error of dw in binary32, norm against norm, is that of rounding x_hat
    to dy's type (uniform within half an ulp of a value that is itself spread over its binade: 0.29 ulp at
    most), and what 16-bit results add by their own rounding is no more than as much again."""
    from paper_2002_00104_b200 import pwlq
    dt = TYPES[dtype]
    dy, saved = _case(8192, 512, 512, dt)
    want = dy.double().t() @ held64(saved)
    ulp = 2 * HALF_ULP[dt]

    def error(dw):
        return float((dw.double() - want).norm() / want.norm())

    assert error(pwlq.act8_weight_grad(dy, saved, dtype=torch.float32)) <= 0.29 * ulp
    assert error(pwlq.act8_weight_grad(dy, saved)) <= 2 ** 0.5 * 0.29 * ulp
