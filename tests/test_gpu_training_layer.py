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


def _layers():
    """(name, function of leaves, leaves) for each autograd function."""
    from paper_2002_00104_b200 import training
    settings = training.Checkpoints(group=64, ratio=0.4375)
    inputs, _ = _norm_inputs(rows=512, cols=1024)
    x, w = _rand(7, 512, 1024).requires_grad_(), _rand(8, 256, 1024, scale=0.03).requires_grad_()
    return [("linear", lambda *t: training.linear(*t, settings), [x, w]),
            ("silu", lambda t: training.silu(t, settings), [x]),
            ("block_norm", lambda *t: sum(training.block_norm(*t, gate_tokens=171, settings=settings)), inputs)]


@pytest.mark.parametrize("which", range(3), ids=["linear", "silu", "block_norm"])
def test_checkpoints_are_released_when_backward_has_used_them(which):
    """The output, and with it the graph, lives on; a byte per value of x does not."""
    _, layer, leaves = _layers()[which]
    out = layer(*leaves)
    seed = torch.ones_like(out)
    torch.autograd.grad(out, leaves, seed)        # the libraries' own workspaces
    del out
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    out = layer(*leaves)
    with_graph = torch.cuda.memory_allocated()
    assert with_graph - before >= out.numel() * 2 + 512 * 1024
    grads = torch.autograd.grad(out, leaves, seed)
    del grads
    assert torch.cuda.memory_allocated() - before < out.numel() * 2 + 4096
    with pytest.raises(RuntimeError, match="second time"):
        torch.autograd.grad(out, leaves, seed)


@pytest.mark.parametrize("which", range(3), ids=["linear", "silu", "block_norm"])
def test_a_retained_graph_and_saved_tensor_hooks(which):
    _, layer, leaves = _layers()[which]
    out = layer(*leaves)
    seed = torch.ones_like(out)
    want = torch.autograd.grad(out, leaves, seed, retain_graph=True)
    again = torch.autograd.grad(out, leaves, seed)
    packed = []

    def to_host(t):
        packed.append(t.dtype)
        return t.cpu()

    with torch.autograd.graph.saved_tensors_hooks(to_host, lambda t: t.cuda()):
        out = layer(*leaves)
    assert torch.uint8 in packed
    moved = torch.autograd.grad(out, leaves, seed)
    for a, b, c in zip(want, again, moved):
        assert torch.equal(a, b) and torch.equal(a, c)


def test_memory_of_another_size_is_refused():
    from paper_2002_00104_b200 import pwlq
    memory, layout = pwlq.act8_encode(_rand(1, 4, 64)).detached()
    assert layout.attached(memory).codes.data_ptr() == memory.data_ptr()
    for bad in (memory[:-1], memory.view(torch.int32), memory.repeat(2)[::2]):
        with pytest.raises(ValueError):
            layout.attached(bad)
    with pytest.raises(ValueError):
        pwlq.Act8(torch.zeros(4, 64, dtype=torch.uint8, device="cuda"), torch.zeros(4, 1, device="cuda"), 64, 64,
                  0.5).detached()


@pytest.mark.parametrize("which", range(3), ids=["linear", "silu", "block_norm"])
def test_second_derivatives_are_refused(which):
    _, layer, leaves = _layers()[which]
    out = layer(*leaves)
    first = torch.autograd.grad(out.float().square().sum(), leaves, create_graph=True)
    second = sum(g.float().square().sum() for g in first)
    with pytest.raises(RuntimeError):
        torch.autograd.grad(second, leaves, retain_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        second.backward()


def test_linear_refuses_types_without_a_weight_gradient_in_the_forward_pass():
    from paper_2002_00104_b200 import training
    x, w = _rand(1, 8, 64, dtype=torch.float32), _rand(2, 32, 64, dtype=torch.float32)
    settings = training.Checkpoints()
    with pytest.raises(ValueError, match="bfloat16 or float16"):
        training.linear(x, w.requires_grad_(), settings)
    with torch.no_grad():                                   # no gradient will be asked for
        y = training.linear(x, w, settings)
    assert torch.equal(y, x @ w.detach().t())
    x.requires_grad_()
    y = training.linear(x, w.detach(), settings)            # a frozen weight
    dx, = torch.autograd.grad(y.sum(), x)
    assert torch.allclose(dx, w.detach().sum(0).expand(8, 64), rtol=1e-5, atol=1e-5)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_block_norm_without_the_outer_norm(dtype):
    from paper_2002_00104_b200 import pwlq, training
    (x, f, _, post, gate), d = _norm_inputs(dtype=dtype)
    r, h = training.block_norm(x, f, None, post, gate, gate_tokens=16)
    assert h is None
    got = torch.autograd.grad(r, (x, f, post, gate), d)
    with torch.no_grad():
        r2, _, saved = pwlq.block_norm(x, f, None, post, gate, gate_tokens=16, save=(128, 0.5))
        want = pwlq.block_norm_backward(saved, dr=d)
    assert torch.equal(r, r2)
    for g, k in zip(got, ("dx", "df", "dpost", "dgate")):
        assert torch.equal(g, want[k])


@pytest.mark.parametrize("used", ["r", "h", "both"])
def test_block_norm_with_one_output_used(used):
    from paper_2002_00104_b200 import pwlq, training
    leaves, d = _norm_inputs()
    r, h = training.block_norm(*leaves, gate_tokens=16)
    outs = [t for t, n in ((r, "r"), (h, "h")) if used in (n, "both")]
    got = torch.autograd.grad(outs, leaves, [d] * len(outs))
    with torch.no_grad():
        _, _, saved = pwlq.block_norm(*leaves, gate_tokens=16, save=(128, 0.5))
        want = pwlq.block_norm_backward(saved, torch.zeros_like(d) if used == "r" else d,
                                        None if used == "h" else d)
    for g, k in zip(got, ("dx", "df", "dpre", "dpost", "dgate")):
        assert torch.equal(g, want[k])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 77), (600, 1024)])
def test_silu_gradient_is_rounded_once(rows, cols, dtype):
    """Against dy * s * (1 + x * (1 - s)) in binary64 at the checkpoint's values.  In binary32 s is good
    to about 8 roundings (exp to 2 ulp, a sum, a quotient), 1 - s to 9 of 1, the factor therefore to 12
    of 1 + |x|, and the products with s and dy add 10."""
    from paper_2002_00104_b200 import pwlq, training
    from train_util import U, check, held64
    settings = training.Checkpoints(group=64, ratio=0.4375)
    x = _rand(rows, rows, cols, scale=3.0, dtype=dtype).requires_grad_()
    dy = _rand(cols, rows, cols, dtype=dtype)
    y = training.silu(x, settings)
    assert torch.equal(y, torch.nn.functional.silu(x))
    dx, = torch.autograd.grad(y, x, dy)
    v = held64(pwlq.act8_encode(x.detach(), 64, 0.4375))
    s = torch.sigmoid(v)
    bound = 24 * U * dy.double().abs() * s * (1 + v.abs())
    check(dx, dy.double() * s * (1 + v * (1 - s)), bound, "dx")
    # a gradient that is broadcast or transposed
    for d in (dy[:1].expand(rows, cols), dy.t().contiguous().t()):
        y = training.silu(x, settings)
        dx, = torch.autograd.grad(y, x, d)
        check(dx, d.double() * s * (1 + v * (1 - s)), 24 * U * d.double().abs() * s * (1 + v.abs()), "dx")


def test_group_lengths_beyond_32_bits_are_refused():
    from paper_2002_00104_b200 import pwlq
    x = _rand(1, 4, 512)
    saved = pwlq.act8_encode(x)
    wrong = pwlq.Act8(saved.codes, saved.ranges[:, :1].contiguous(), 512, 2 ** 32 + 64, 0.5)
    for call in (lambda: pwlq.act8_encode(x, group=2 ** 32 + 64), lambda: pwlq.act8_decode(wrong),
                 lambda: pwlq.act8_weight_grad(x, wrong),
                 lambda: pwlq.block_norm(x, pre_weight=x[0].contiguous(), save=(2 ** 32 + 64, 0.5))):
        with pytest.raises(pwlq.PwlqError) as e:
            call()
        assert e.value.status == pwlq.ERR_INVALID_ARG


def test_gates_of_no_tokens_are_refused():
    from paper_2002_00104_b200 import pwlq
    (x, f, pre, post, gate), _ = _norm_inputs()
    with torch.no_grad():
        for tokens in (0, -1, -2 ** 63):
            with pytest.raises(pwlq.PwlqError) as e:
                pwlq.block_norm(x, f, pre, post, gate, gate_tokens=tokens)
            assert e.value.status == pwlq.ERR_INVALID_ARG
            pwlq.block_norm(x, f, pre, post, gate_tokens=tokens)         # there is no gate
        want = pwlq.block_norm(x, f, pre, post, gate, gate_tokens=16)
        got = pwlq.block_norm(x, f, pre, post, gate)                     # 48 rows over 3 gates
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_best_ratio_of_rows_shorter_than_a_group():
    from paper_2002_00104_b200 import training
    x = _rand(3, 300, 96, dtype=torch.float32) ** 3
    assert training.best_ratio(x, group=128) == training.best_ratio(x, group=96)
    assert training.best_ratio(x[:1, :1]) < 1
    for bad in (x[:0], x[:, :0]):
        with pytest.raises(ValueError):
            training.best_ratio(bad)
    with pytest.raises(ValueError):
        training.best_ratio(x, candidates=1)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,cols,outputs", [(1, 8, 3), (77, 200, 130), (600, 1024, 515)])
def test_linear_against_the_formula(rows, cols, outputs, dtype):
    """dx = dy W as PyTorch has it; dw = dy^T x_hat at the checkpoint's values (the bounds of the weight
    gradient's own tests: half an ulp of x_hat, sums of 16 products at a time, the result's rounding)."""
    from paper_2002_00104_b200 import pwlq, training
    from train_util import HALF_ULP, SUBNORMAL, check, held64
    settings = training.Checkpoints(group=32, ratio=0.375)
    x = _rand(rows, rows, cols, dtype=dtype).requires_grad_()
    w = _rand(cols, outputs, cols, scale=0.05, dtype=dtype).requires_grad_()
    dy = _rand(outputs, rows, outputs, scale=0.1, dtype=dtype)
    held, w64 = held64(pwlq.act8_encode(x.detach(), 32, 0.375)), w.detach().double()
    for d in (dy, dy[:1].expand(rows, outputs), dy.t().contiguous().t()):
        y = training.linear(x, w, settings)
        assert torch.equal(y, x @ w.t())
        dx, dw = torch.autograd.grad(y, (x, w), d)
        assert torch.equal(dx, d @ w.detach())
        want, mag = d.double().t() @ held, d.double().abs().t() @ held.abs()
        slack = (2.0 ** -22 * (rows / 16 + 25) + HALF_ULP[dtype]) * mag
        check(dw, want, slack + SUBNORMAL[dtype] * d.double().abs().sum(0)[:, None], "dw")


# f: block output, o: norm after it, g: gate, p: norm before the next block
@pytest.mark.parametrize("kind", ["fogp", "fop", "fgp", "fp", "p", "fog", "fo", "fg"])
@pytest.mark.parametrize("dtype,wtype", [(torch.bfloat16, torch.bfloat16), (torch.float16, torch.float32),
                                         (torch.float32, torch.float32)])
def test_block_norm_is_the_calls_it_is_made_of(kind, dtype, wtype):
    from paper_2002_00104_b200 import pwlq, training
    rows, cols = 60, 304
    x = _rand(1, rows, cols, dtype=dtype)
    f = _rand(2, rows, cols, dtype=dtype) if "f" in kind else None
    post = 1 + _rand(3, cols, scale=0.2, dtype=wtype) if "o" in kind else None
    gate = _rand(4, 4, cols, scale=0.5, dtype=wtype) if "g" in kind else None
    pre = 1 + _rand(5, cols, scale=0.2, dtype=wtype) if "p" in kind else None
    dr, dh = _rand(6, rows, cols, scale=0.1, dtype=dtype), _rand(7, rows, cols, scale=0.1, dtype=dtype)
    settings = training.Checkpoints(group=64, ratio=0.4375)
    want_r, want_h, saved = pwlq.block_norm(x, f, pre, post, gate, residual_scale=0.5, eps=1e-5, save=(64, 0.4375))
    want = pwlq.block_norm_backward(saved, dh if pre is not None else None, dr)
    leaves = [t.requires_grad_() for t in (x, f, pre, post, gate) if t is not None]
    r, h = training.block_norm(x, f, pre, post, gate, residual_scale=0.5, eps=1e-5, settings=settings)
    assert torch.equal(r, want_r) and (h is None) == (want_h is None) and (h is None or torch.equal(h, want_h))
    outs, seeds = ([r, h], [dr, dh]) if h is not None else ([r], [dr])
    got = torch.autograd.grad(outs, leaves, seeds)
    for g, w in zip(got, [v for v in want.values() if v is not None], strict=True):
        assert torch.equal(g, w)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("seed", [0, 1])
def test_gradients_of_a_network_in_either_type(dtype, seed):
    """The example's network against the same in PyTorch, in bf16 and fp16 (the reasons for 5 % are those of
    the example's own test; fp16 rounds less)."""
    import os
    import sys
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import train_act8
    from paper_2002_00104_b200 import training
    dt = getattr(torch, dtype)
    x, t = _rand(seed, 512, 256, dtype=dt), _rand(seed + 10, 512, 256, dtype=torch.float32)
    settings = training.Checkpoints(group=64, ratio=0.5)

    def grads(forward):
        p = {k: [v.to(dt) for v in vs] for k, vs in train_act8.parameters(256, 2, seed).items()}
        leaves = [v.requires_grad_() for group in p.values() for v in group]
        return torch.autograd.grad((forward(p, x).float() * t).sum(), leaves)

    for g, w in zip(grads(lambda p, v: train_act8.forward_act8(p, v, settings)), grads(train_act8.forward_plain)):
        assert g.dtype == w.dtype == dt
        assert (g.float() - w.float()).norm() <= 0.05 * w.float().norm()
