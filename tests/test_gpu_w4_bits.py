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


def _thirds(seed, rows, cols, top):
    """Values 0, +-m / 3, +-2 m / 3, +-m, with m = 3 * top in every group of 32."""
    g = torch.Generator().manual_seed(seed)
    w = torch.randint(-3, 4, (rows, cols), generator=g).float()
    w[:, ::32] = 3.0
    return w * top


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("tokens,rows,cols,group", [(1, 40, 256, 32), (3, 40, 301, 64), (8, 4096, 8192, 128), (9, 48, 384, 256),
                                                    (5, 33600, 300, 128), (70, 20, 128, 64)])
def test_the_largest_activations(dtype, tokens, rows, cols, group):
    """Values up to the largest bf16 ones, whose sum before the scales lies behind binary32's range, and the result
    far within it."""
    from paper_2002_00104_b200 import pwlq
    w = _thirds(rows, rows, cols, 2.0 ** -16)
    x = torch.tensor([1.0, -1.0, 1.9921875, -1.9921875, 0.0])[torch.randint(0, 5, (tokens, cols), generator=torch.Generator().manual_seed(cols))]
    x = (x.double() * 2.0 ** 127).float()
    assert torch.isfinite(x).all() and torch.equal(x.bfloat16().float(), x)
    y = pwlq.w4_linear(x.to(TYPES[dtype]).cuda(), _pack(w, group)).cpu()
    assert torch.equal(y, (x.double() @ w.double().t()).to(y.dtype))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("tokens,rows,cols,group", [(1, 40, 256, 32), (3, 40, 301, 64), (9, 48, 384, 256), (5, 33600, 300, 128)])
def test_the_smallest_activations(dtype, tokens, rows, cols, group):
    """Values at the lower end of the normal numbers, products of which with the levels alone are below it."""
    from paper_2002_00104_b200 import pwlq
    w = _thirds(rows, rows, cols, 2.0 ** 30)
    x = torch.randint(-3, 4, (tokens, cols), generator=torch.Generator().manual_seed(cols)).float() * 2.0 ** -126
    y = pwlq.w4_linear(x.to(TYPES[dtype]).cuda(), _pack(w, group)).cpu()
    assert torch.equal(y, (x.double() @ w.double().t()).to(y.dtype))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("tokens,features", [(1, 64), (2, 4096), (20, 70)])
def test_the_largest_values_in_a_layer(dtype, tokens, features):
    """The same in both products: of values of 2^127, and of 27 * 2^120 between them."""
    hidden = 40
    up, down = torch.zeros(2 * hidden, features), _thirds(features, features, hidden, 2.0 ** -40)
    x = torch.zeros(tokens, features)
    x[:, :3] = 2.0 ** 127
    up[:hidden, :3] = 3 * 2.0 ** -98                     # gate 9 * 2^29: its sigmoid is 1
    up[hidden:, 0] = 3 * 2.0 ** -36                      # up 3 * 2^91
    want = (torch.full((hidden,), 27.0 * 2.0 ** 120).double() @ down.double().t()).expand(tokens, -1)
    y = _one_expert(up, down, x, TYPES[dtype])
    assert torch.equal(y, want.to(y.dtype))


@pytest.mark.parametrize("tokens,features", [(1, 64), (2, 4096), (7, 70), (20, 64), (33, 130)])
def test_all_bits_of_binary32_tokens_in_a_layer(tokens, features):
    """Tokens that differ in their 24th bit: gate and up sums of two that cancel are all that is left of them."""
    hidden = 40
    up, down = torch.zeros(2 * hidden, features), torch.zeros(features, hidden)
    x = torch.zeros(tokens, features)
    x[:, 0] = 1.0 + 2.0 ** -12 + 2.0 ** -23
    x[:, 1] = 1.0 + 2.0 ** -12
    up[0, 0], up[0, 1] = 3 * 2.0 ** 30, -3 * 2.0 ** 30   # gate 3 * 2^7: its sigmoid is 1
    up[hidden, 0], up[hidden, 1] = 3 * 2.0 ** 10, -3 * 2.0 ** 10     # up 3 * 2^-13
    c = 3.0 * 2.0 ** torch.randint(-3, 4, (features,), generator=torch.Generator().manual_seed(features)).float()
    down[:, 0] = c
    y = _one_expert(up, down, x, torch.float32)
    assert torch.equal(y, (c * 384 * 3 * 2.0 ** -13).expand(tokens, -1))
