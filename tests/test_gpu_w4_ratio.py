"""The breakpoint of several weight matrices at once."""
import pytest
import torch

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a CUDA device")]


@pytest.mark.parametrize("matrices,rows,cols,group", [(1, 64, 96, 64), (6, 40, 96, 64), (3, 130, 260, 128), (4, 64, 100, 128), (5, 7, 512, 32)])
def test_best_ratio_of_several_matrices(matrices, rows, cols, group):
    """That of all their rows, in the groups in which they are packed."""
    from paper_2002_00104_b200 import pwlq, training
    g = torch.Generator("cuda").manual_seed(rows)
    w = torch.randn(matrices, rows, cols, generator=g, device="cuda") ** 3
    whole = cols // group * group
    w[..., :whole] = torch.rand(matrices, rows, whole, generator=g, device="cuda") - 0.5      # and the rest unlike them
    best = training.best_ratio(w, group, 64, bits=3)
    assert best == training.best_ratio(w.flatten(0, 1), group, 64, bits=3)
    kept = w[..., :whole or cols]
    error = {r: float((pwlq.w4_decode(pwlq.w4_encode(kept.contiguous(), group=group, ratio=r)) - kept).square().sum())
             for r in (best, 0.125, 0.875)}
    assert error[best] <= min(error.values()) * 1.01     # the search takes ranges in 32 bits, the format in 8


def test_shapes_that_are_no_matrices():
    from paper_2002_00104_b200 import training
    x = torch.ones(64, device="cuda")
    for bad in (x, x[0], x.view(2, 2, 2, 8), x.view(8, 8)[:0], x.view(1, 8, 8)[:, :, :0]):
        with pytest.raises(ValueError):
            training.best_ratio(bad, 32)
