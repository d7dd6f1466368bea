"""The autograd functions: what they keep, what they refuse, and their gradients."""
import pytest
import torch

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a CUDA device")]


def _rand(seed, *shape, scale=1.0, dtype=torch.bfloat16):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)


def _norm_inputs(rows=48, cols=256, dtype=torch.bfloat16):
    x, f = _rand(1, rows, cols, dtype=dtype), _rand(2, rows, cols, dtype=dtype)
    pre, post = (1 + _rand(s, cols, scale=0.2, dtype=dtype) for s in (3, 4))
    gate = _rand(5, 3, cols, scale=0.5, dtype=dtype)
    return [t.requires_grad_() for t in (x, f, pre, post, gate)], _rand(6, rows, cols, scale=0.1, dtype=dtype)


@pytest.mark.parametrize("layer", ["calls", "autograd"])
def test_weights_are_read_where_they_are_when_backward_runs(layer):
    """A parameter whose storage is replaced between forward and backward (memory freed and gathered
    again): the old memory is overwritten here, and the gradients stay the same."""
    from paper_2002_00104_b200 import pwlq, training
    (x, f, pre, post, gate), d = _norm_inputs()
    results = []
    for moved in (False, True):
        if layer == "autograd":
            r, h = training.block_norm(x, f, pre, post, gate, gate_tokens=16)
        else:
            with torch.no_grad():
                _, _, saved = pwlq.block_norm(x, f, pre, post, gate, gate_tokens=16, save=(128, 0.5))
        if moved:
            for w in (pre, post, gate):
                old = w.data
                w.data = old.clone()
                old.fill_(7.0)
        if layer == "autograd":
            results.append(torch.autograd.grad((r.float() + h.float()).mul(d.float()).sum(),
                                               (x, f, pre, post, gate)))
        else:
            results.append(list(pwlq.block_norm_backward(saved, d, d).values()))
    for a, b in zip(*results):
        assert torch.equal(a, b)


@pytest.mark.parametrize("which", [2, 3, 4])
def test_a_weight_changed_in_place_after_the_forward_pass_is_refused(which):
    from paper_2002_00104_b200 import training
    inputs, d = _norm_inputs()
    r, h = training.block_norm(*inputs, gate_tokens=16)
    with torch.no_grad():
        inputs[which].mul_(2)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        torch.autograd.grad((h.float() * d.float()).sum(), inputs)


def test_kept_memory_of_other_weights_is_refused():
    from paper_2002_00104_b200 import pwlq
    (x, f, pre, post, gate), d = _norm_inputs()
    with torch.no_grad():
        _, _, saved = pwlq.block_norm(x, f, pre, post, gate, gate_tokens=16, save=(128, 0.5))
    for name, bad in (("pre_weight", pre.float()), ("pre_weight", pre[:255]), ("post_weight", post.cpu()),
                      ("gate", gate[:2]), ("gate", gate[:, :255])):
        good = getattr(saved, name)
        setattr(saved, name, bad.detach())
        with pytest.raises(ValueError):
            pwlq.block_norm_backward(saved, d, d)
        setattr(saved, name, good)
    saved.pre_weight = None
    with pytest.raises(ValueError):
        pwlq.block_norm_backward(saved, None, d)
