"""The block norm's backward pass on values near the end of their type's range."""
import pytest
import torch

from train_util import TYPES, U, backward64, check, held64

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a CUDA device")]


# rows a few lanes wide; rings; rings on rows off their alignment; threads that load for themselves; pairs;
# sums in shared memory
@pytest.mark.parametrize("rows,cols", [(40, 48), (64, 1040), (64, 1283), (30, 4100), (20, 8704), (20, 8399)])
@pytest.mark.parametrize("dtype,wtype", [("bf16", "bf16"), ("bf16", "fp32"), ("fp32", "fp32")])
@pytest.mark.parametrize("ratio", [0.4375, 1.0])
@pytest.mark.parametrize("every", [1000, 7])
def test_gate_gradients_of_values_up_to_the_largest(rows, cols, dtype, wtype, ratio, every):
    """A block output up to 3.3e38 that enters through a gate alone: dgate = sum of dr * F is in range.  Each
    held value is within 6 roundings of its group's range (a piece's line: its two constants of 2 roundings
    each, one fused operation, for a value of at most the range), and is summed over at most `rows` rows."""
    from paper_2002_00104_b200 import pwlq
    dt, wt, group = TYPES[dtype], TYPES[wtype], 64
    g = torch.Generator(device="cuda")
    g.manual_seed(rows * cols)
    f = torch.rand(rows, cols, generator=g, device="cuda") * 2 - 1
    f *= torch.tensor([3.3e38, 1.0, 1.1e38, 3.0e30], device="cuda").repeat(rows)[:rows, None]
    f = f.to(dt)
    x = torch.zeros_like(f)
    gate = (torch.rand(-(-rows // every), cols, generator=g, device="cuda") * 0.5).to(wt)
    dr = (torch.randn(rows, cols, generator=g, device="cuda") * 0.01).to(dt)
    r, _, saved = pwlq.block_norm(x, f, gate=gate, gate_tokens=every, save=(group, ratio))
    assert torch.isfinite(r).all()
    got = pwlq.block_norm_backward(saved, dr=dr)
    F = held64(saved.f)
    want, mag = backward64(None, F, None, None, None, dr.double(), None, None, gate.double(), every, 1.0, 0.0)
    m = saved.f.ranges.double().repeat_interleave(group, dim=1)[:, :cols]
    _, size = backward64(None, m, None, None, None, dr.double(), None, None, gate.double(), every, 1.0, 0.0)
    check(got["df"], want["df"], 4 * U * mag["df"], "df")
    check(got["dgate"], want["dgate"], U * (6 + rows) * size["dgate"], "dgate")


@pytest.mark.parametrize("at", [1, 3, 7])
def test_first_rows_off_their_alignment_are_followed_by_others_in_their_place(at):
    """Gapless rows of odd length from an odd address: the first row's beginning and the last one's end are
    moved value by value, and further rows take the same bytes of shared memory.  The same results as from an
    aligned address."""
    from paper_2002_00104_b200 import pwlq
    rows, cols = 5000, 1283
    g = torch.Generator(device="cuda")
    g.manual_seed(at)

    def both(seed):
        store = torch.randn(at + rows * cols, generator=g, device="cuda").bfloat16()
        odd = store[at:].view(rows, cols)
        return odd, odd.clone()

    x, f, dh, dr = (both(i) for i in range(4))
    w = torch.rand(cols, generator=g, device="cuda").bfloat16()
    results = []
    for i in range(2):
        r, h, saved = pwlq.block_norm(x[i], f[i], w, w, save=(64, 0.5))
        results.append([r, h, *(v for v in pwlq.block_norm_backward(saved, dh[i], dr[i]).values() if v is not None)])
    for a, b in zip(*results):
        assert torch.equal(a, b)
    assert pwlq.device_status() == 0
