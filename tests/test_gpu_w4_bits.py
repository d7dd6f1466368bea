"""Products with 4-bit weights: which bits and which range reach the result.  Every case's sums are exact in
binary32 in any order, so that results are compared for equality."""
import pytest
import torch

from w4_util import TYPES

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a CUDA device")]


def _pack(w, group=32, paired=False):
    """w of values 0, m / 3, 2 m / 3, m in every group, m of 3 times a power of two: held as they are."""
    from paper_2002_00104_b200 import pwlq
    packed = pwlq.w4_encode(w.cuda(), group=group, ratio=1.0, paired=paired)
    assert torch.equal(pwlq.w4_decode(packed).cpu(), w)
    return packed


def _one_expert(up, down, x, dtype):
    """The layer of a single expert, whose weight is 1."""
    from paper_2002_00104_b200 import pwlq
    router = torch.zeros(1, x.shape[1], dtype=dtype, device="cuda")
    return pwlq.w4_moe(x.to(dtype).cuda(), router, _pack(up[None], paired=True), _pack(down[None]), 1).cpu()


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("tokens,features", [(1, 64), (1, 4096), (7, 70), (8, 4096), (20, 64), (33, 130)])
def test_all_bits_between_the_products(dtype, tokens, features):
    """h0 and h1 are 24-bit numbers that differ in the last two bits; h0 - h1 is all that is left of them."""
    hidden = 40
    up, down = torch.zeros(2 * hidden, features), torch.zeros(features, hidden)
    x = torch.zeros(tokens, features)
    x[:, 0], x[:, 1], x[:, 2], x[:, 33] = 32.0, 1.0, 2.0 ** -9, 2.0 ** -13
    up[:2, 0] = 3.0                                      # gate 96: its sigmoid is 1 in binary32
    up[hidden:hidden + 2, 1:3] = 3.0                     # up 3 + 3 * 2^-9, and 2^-20 more in the first row
    up[hidden, 33], up[hidden, 34] = 2.0 ** -7, 3 * 2.0 ** -7
    c = 3.0 * 2.0 ** torch.randint(-3, 4, (features,), generator=torch.Generator().manual_seed(features)).float()
    down[:, 0], down[:, 1] = c, -c
    y = _one_expert(up, down, x, TYPES[dtype])
    assert torch.equal(y.float(), (c * 96 * 2.0 ** -20).expand(tokens, -1))
