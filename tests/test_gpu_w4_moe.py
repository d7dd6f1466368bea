"""The mixture-of-experts layer on 4-bit weights: choice, products, and what a user runs them in."""
import threading

import numpy as np
import pytest
import torch

import w4_util as U
from w4_util import TYPES

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a CUDA device")]


def _t(seed, *shape, dtype=torch.float32, scale=1.0):
    rng = np.random.default_rng(seed)
    return torch.from_numpy((rng.standard_t(5, shape) * scale).astype(np.float32)).to(dtype)


def _layer(seed, experts, features, hidden, dtype, group=64, ratio=0.4375, router_dtype=None):
    from paper_2002_00104_b200 import pwlq
    up = _t(seed, experts, 2 * hidden, features, dtype=dtype, scale=features ** -0.5)
    down = _t(seed + 1, experts, features, hidden, dtype=dtype, scale=hidden ** -0.5)
    router = _t(seed + 2, experts, features, dtype=router_dtype or dtype, scale=features ** -0.5)
    s = {"router": router.cuda(), "up": pwlq.w4_encode(up.cuda(), group=group, ratio=ratio, paired=True),
         "down": pwlq.w4_encode(down.cuda(), group=group, ratio=ratio)}
    return s, U.held(up, group, ratio), U.held(down, group, ratio)


def _run(s, x, top, **kw):
    from paper_2002_00104_b200 import pwlq
    return pwlq.w4_moe(x, s["router"], s["up"], s["down"], top, **kw)


def _check(s, up, down, x, top, normalize):
    y, experts, weights = _run(s, x.cuda(), top, normalize=normalize, want_routing=True)
    want, bound, e, w = U.moe(x, s["router"], up, down, top, normalize)
    assert torch.equal(experts.cpu().long(), e)
    # exp, a sum of at most 1024 terms and a quotient in binary32
    assert bool(((weights.cpu().double() - w).abs() <= 2.0 ** -20 * w + 1e-30).all())
    U.check(y, want, bound)
    assert torch.equal(y, _run(s, x.cuda(), top, normalize=normalize))
    return y


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("tokens,features,hidden,experts,top,group,normalize", [
    (1, 64, 64, 4, 2, 32, True), (1, 256, 128, 64, 8, 128, True), (1, 1, 1, 1, 1, 64, False), (2, 300, 70, 3, 3, 64, False),
    (5, 129, 515, 17, 3, 32, False), (8, 512, 96, 8, 2, 256, True), (9, 130, 40, 5, 4, 64, True), (16, 384, 200, 100, 32, 64, False),
    (33, 96, 129, 2, 1, 128, True), (64, 256, 64, 32, 4, 64, True), (64, 72, 24, 1024, 5, 32, True),
    (40, 4096, 24, 48, 4, 64, True), (3, 4100, 2056, 2, 1, 128, True), (8, 4096, 2050, 2, 2, 32, False)])
def test_layers(dtype, tokens, features, hidden, experts, top, group, normalize):
    dt = TYPES[dtype]
    s, up, down = _layer(tokens * 31 + features, experts, features, hidden, dt, group)
    _check(s, up, down, _t(tokens, tokens, features, dtype=dt), top, normalize)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_a_router_in_binary32(dtype):
    s, up, down = _layer(3, 16, 200, 64, TYPES[dtype], router_dtype=torch.float32)
    _check(s, up, down, _t(5, 7, 200, dtype=TYPES[dtype]), 4, True)


@pytest.mark.parametrize("tokens", [8, 9, 64])
def test_all_tokens_at_the_same_experts(tokens):
    """An expert with every token and others with none."""
    s, up, down = _layer(11, 12, 160, 72, torch.bfloat16)
    x = _t(12, tokens, 160, dtype=torch.bfloat16)
    x[:, 0] = 8.0
    s["router"][:, 0] = 0.0
    s["router"][[7, 2], 0] = torch.tensor([8.0, 6.0], device="cuda").bfloat16()
    _check(s, up, down, x, 2, True)


def test_equal_scores_go_to_the_lowest_index():
    s, up, down = _layer(21, 40, 64, 32, torch.bfloat16)
    s["router"][:] = s["router"][0]
    s["router"][17] *= 2
    x = _t(22, 6, 64, dtype=torch.bfloat16)
    x[3] = 0.0                                           # every score is 0
    _, experts, _ = _run(s, x.cuda(), 5, want_routing=True)
    assert torch.equal(experts[3].cpu(), torch.arange(5, dtype=torch.int32))
    _check(s, up, down, x, 5, False)


def test_scores_that_differ_in_their_last_bits():
    """Sums in another order, or in binary32, would choose otherwise: terms of 2^12 that cancel leave 2^-13."""
    from paper_2002_00104_b200 import pwlq
    experts, features = 16, 4096
    router = torch.zeros(experts, features)
    rng = np.random.default_rng(5)
    for e in range(experts):
        place = rng.permutation(features)
        router[e, place[:1000]] = 64.0
        router[e, place[1000:2000]] = -64.0
        router[e, place[2000]] = float(e % 7 + 1) * 2.0 ** -19
    s, up, down = _layer(31, experts, features, 16, torch.float32)
    s["router"] = router.cuda()
    x = torch.full((3, features), 64.0) * torch.tensor([[1.0], [0.5], [-1.0]])
    _, got, _ = pwlq.w4_moe(x.cuda(), s["router"], s["up"], s["down"], 6, want_routing=True)
    assert torch.equal(got.cpu().long(), U.route(x, router, 6, True)[0])


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("tokens", [6, 20])
def test_infinities_and_nan_stay_with_their_tokens(dtype, tokens):
    dt = TYPES[dtype]
    s, up, down = _layer(41, 8, 200, 96, dt)
    x = _t(42, tokens, 200, dtype=dt).cuda()
    clean = _run(s, x, 3)
    x[1, 5], x[4, 199] = float("nan"), float("inf")
    y, experts, weights = _run(s, x, 3, want_routing=True)
    assert torch.isnan(y[1]).all() and torch.isnan(y[4]).all() and torch.isnan(weights[1]).all()
    assert torch.equal(experts[1].cpu(), torch.arange(3, dtype=torch.int32))
    keep = [t for t in range(tokens) if t not in (1, 4)]
    assert torch.equal(y[keep], clean[keep])


def test_a_nan_score_is_chosen_and_seen():
    s, _, _ = _layer(51, 8, 64, 32, torch.bfloat16)
    s["router"][6, 0] = float("nan")
    y, experts, weights = _run(s, _t(52, 2, 64, dtype=torch.bfloat16).cuda(), 2, want_routing=True)
    assert (experts[:, 0] == 6).all() and torch.isnan(weights).all() and torch.isnan(y).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("tokens", [3, 30])
def test_rows_off_their_alignment_in_place_and_around(dtype, tokens):
    dt = TYPES[dtype]
    s, up, down = _layer(61, 6, 129, 70, dt)
    wide = torch.full((tokens, 140), 7.0, dtype=dt, device="cuda")
    wide[:, 5:134] = _t(62, tokens, 129, dtype=dt).cuda()
    x = wide[:, 5:134]
    router = torch.full((6, 133), float("nan"), dtype=dt, device="cuda")
    router[:, 1:130] = s["router"]
    s["router"] = router[:, 1:130]
    want = _check(s, up, down, x.cpu(), 2, True)
    assert torch.equal(_run(s, x, 2), want)
    assert torch.equal(_run(s, x, 2, out=x), want) and torch.equal(x, want)
    assert (wide[:, :5] == 7).all() and (wide[:, 134:] == 7).all()


def test_values_beyond_fp16_between_the_products():
    """silu(gate) * up up to 2^20: held with binary32's range."""
    from paper_2002_00104_b200 import pwlq
    up = torch.full((1, 32, 64), 2.0 ** 4)
    down = torch.zeros(1, 64, 16)
    down[0, :, 0], down[0, :, 1] = 2.0 ** -8, -2.0 ** -8
    down[0, 3, 1] = 0.0
    s = {"router": torch.zeros(1, 64, device="cuda").half(), "up": pwlq.w4_encode(up.cuda(), group=32, ratio=1.0, paired=True),
         "down": pwlq.w4_encode(down.cuda(), group=32, ratio=1.0)}
    x = torch.ones(1, 64).half()
    want, bound, _, _ = U.moe(x, s["router"], U.held(up, 32, 1.0), U.held(down, 32, 1.0), 1, True)
    assert float(want[0, 3]) > 4000 and float(U.linear(x, U.held(up[0], 32, 1.0), True)[0].max()) > 2 ** 19
    U.check(_run(s, x.cuda(), 1), want, bound)


def test_workspaces_and_refusals():
    from paper_2002_00104_b200 import pwlq
    s, _, _ = _layer(71, 8, 128, 64, torch.bfloat16)
    x = _t(72, 4, 128, dtype=torch.bfloat16).cuda()
    need = pwlq.w4_moe_workspace_bytes(4, 2, 128, 64)
    workspace = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    want = _run(s, x, 2)
    assert torch.equal(_run(s, x, 2, workspace=workspace), want)
    assert _run(s, x[:0], 2).shape == (0, 128)
    for bad in (lambda: _run(s, x.float(), 2), lambda: _run(s, x[:, :64], 2), lambda: _run(s, x, 2, out=x[:3]),
                lambda: _run(s, x, 2, workspace=workspace.cpu()), lambda: _run(s, x.cpu(), 2),
                lambda: _run({**s, "up": s["down"]}, x, 2),      # of other columns than x
                lambda: _run({**s, "router": s["router"][:7]}, x, 2), lambda: _run({**s, "router": s["router"].half()}, x, 2),
                lambda: _run(s, x.float().requires_grad_().bfloat16(), 2),
                lambda: _run({**s, "router": s["router"].float().requires_grad_()}, x, 2)):
        with pytest.raises(ValueError):
            bad()
    many = x[:1].expand(65, 128).contiguous()
    for bad, status in ((lambda: _run(s, x, 9), pwlq.ERR_INVALID_ARG), (lambda: _run(s, x, 0), pwlq.ERR_INVALID_ARG),
                        (lambda: _run(s, many, 2), pwlq.ERR_UNSUPPORTED), (lambda: _run(s, x, 33), pwlq.ERR_INVALID_ARG),
                        (lambda: _run(s, x, 2 ** 32 + 2), pwlq.ERR_INVALID_ARG),
                        (lambda: _run({**s, "down": s["up"]}, x, 2), pwlq.ERR_INVALID_ARG),
                        (lambda: _run(s, x, 2, workspace=workspace[:-1]), pwlq.ERR_WORKSPACE)):
        with pytest.raises(pwlq.PwlqError) as e:
            bad()
        assert e.value.status in (status, pwlq.ERR_UNSUPPORTED)


def test_experts_beyond_4_gb():
    """The last of 160 experts lies more than 2^32 bytes into its memory."""
    from paper_2002_00104_b200 import pwlq
    one = _t(81, 2 * 4096, 4096, dtype=torch.bfloat16, scale=0.02).cuda()
    up = pwlq.w4_encode(one.expand(260, -1, -1), paired=True)
    assert up.memory.numel() > 1 << 32
    down = pwlq.w4_encode(_t(82, 1, 4096, 4096, dtype=torch.bfloat16, scale=0.02).cuda().expand(260, -1, -1))
    router = torch.zeros(260, 4096, device="cuda")
    x = _t(83, 2, 4096, dtype=torch.bfloat16).cuda()
    x[:, 0] = 1.0
    y = []
    for e in (0, 259):
        router.zero_()
        router[e, 0] = 1.0
        out, experts, _ = pwlq.w4_moe(x, router, up, down, 1, want_routing=True)
        assert (experts == e).all()
        y.append(out)
    assert torch.equal(*y)
    del one
    last = pwlq.w4_decode(up, dtype=torch.bfloat16)[259]
    assert torch.equal(pwlq.w4_encode(last, paired=True).memory,
                       pwlq.w4_encode(pwlq.w4_decode(up, dtype=torch.bfloat16)[0], paired=True).memory)


# ----------------------------------------------------------------------- a decoding step
def _model(seed, features=256, hidden=384, dtype=torch.float32):
    from paper_2002_00104_b200 import pwlq
    m, _, _ = _layer(seed, 16, features, 64, dtype)
    w = {"attn": _t(seed + 5, features, features, dtype=dtype, scale=features ** -0.5),
         "mlp": _t(seed + 6, 2 * hidden, features, dtype=dtype, scale=features ** -0.5),
         "out": _t(seed + 7, features, hidden, dtype=dtype, scale=hidden ** -0.5)}
    for k, v in w.items():
        m[k] = pwlq.w4_encode(v.cuda(), group=64, ratio=0.4375, paired=k == "mlp")
    for i in range(4):
        m["n%d" % i] = (1 + 0.1 * _t(seed + 10 + i, features, dtype=dtype)).cuda()
    return m


def _step(m, x):
    """Norm, projection, norm, gated block, norm, experts, norm, as a block of a model calls them."""
    from paper_2002_00104_b200 import pwlq
    r, h, _ = pwlq.block_norm(x, None, m["n0"])
    f = pwlq.w4_linear(h, m["attn"])
    r, h, _ = pwlq.block_norm(r, f, m["n1"])
    f = pwlq.w4_linear(pwlq.w4_linear(h, m["mlp"]), m["out"])
    r, h, _ = pwlq.block_norm(r, f, m["n2"])
    f = pwlq.w4_moe(h, m["router"], m["up"], m["down"], 4)
    return pwlq.block_norm(r, f, m["n3"])[1]


def _step_exact(m, x):
    from paper_2002_00104_b200 import pwlq

    def norm(v, w):
        return v * torch.rsqrt(v.square().mean(1, keepdim=True) + 1e-6) * w.double()

    w = {k: pwlq.w4_decode(v).double() for k, v in m.items() if isinstance(v, pwlq.W4)}
    r = x.double()
    r = r + norm(r, m["n0"]) @ w["attn"].t()
    gate, up = (norm(r, m["n1"]) @ w["mlp"].t()).chunk(2, 1)
    r = r + (U.silu(gate) * up) @ w["out"].t()
    h = norm(r, m["n2"])
    scores = h @ m["router"].double().t()
    best, chosen = scores.topk(4, dim=1)
    share = torch.softmax(best, dim=1)
    for t in range(x.shape[0]):
        for j in range(4):
            gate, up = (w["up"][chosen[t, j]] @ h[t]).chunk(2)
            r[t] += share[t, j] * (w["down"][chosen[t, j]] @ (U.silu(gate) * up))
    return norm(r, m["n3"])


@pytest.mark.parametrize("tokens", [1, 5, 33])
def test_a_block_of_all_of_them(tokens):
    m, x = _model(91), _t(92, tokens, 256).cuda()
    y, want = _step(m, x), _step_exact(m, x)
    # nine binary32 results one after another, each within SUM of its magnitudes' sum (at most 30 times its own size)
    assert float((y.double() - want).norm() / want.norm()) <= 9 * 30 * U.SUM


def test_captured_steps_that_share_memory_replayed_on_other_inputs():
    """Two graphs in one memory pool: the workspaces of either are the other's too."""
    m = _model(101, dtype=torch.bfloat16)
    xs = [_t(102, 1, 256, dtype=torch.bfloat16).cuda(), _t(103, 12, 256, dtype=torch.bfloat16).cuda()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for x in xs:
            _step(m, x)
    torch.cuda.current_stream().wait_stream(side)
    graphs, outs = [], []
    for x in xs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, pool=graphs[0].pool() if graphs else None):
            outs.append(_step(m, x))
        graphs.append(g)
    for seed in range(3):
        for i, x in enumerate(xs):
            x.copy_(_t(200 + 10 * seed + i, *x.shape, dtype=torch.bfloat16))
            graphs[i].replay()
            assert torch.equal(outs[i], _step(m, x))


@pytest.mark.parametrize("threads", [False, True])
def test_steps_side_by_side(threads):
    models = [_model(300 + 20 * i, dtype=torch.bfloat16) for i in range(3)]
    xs = [_t(400 + i, n, 256, dtype=torch.bfloat16).cuda() for i, n in enumerate((1, 6, 40))]
    want = [_step(m, x) for m, x in zip(models, xs)]
    streams = [torch.cuda.Stream() for _ in xs]
    got = [None] * len(xs)
    torch.cuda.synchronize()

    def work(i, times):
        torch.cuda.set_device(0)
        with torch.cuda.stream(streams[i]):
            for _ in range(times):
                got[i] = _step(models[i], xs[i])

    if threads:
        workers = [threading.Thread(target=work, args=(i, 20)) for i in range(len(xs))]
        for t in workers:
            t.start()
        for t in workers:
            t.join()
    else:
        for _ in range(20):
            for i in range(len(xs)):
                work(i, 1)
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_a_stream_of_the_caller_s_choice():
    from paper_2002_00104_b200 import pwlq
    s, _, _ = _layer(501, 8, 128, 64, torch.bfloat16)
    x = _t(502, 4, 128, dtype=torch.bfloat16).cuda()
    w = _t(503, 64, 128, dtype=torch.bfloat16).cuda()
    want = pwlq.w4_linear(x, pwlq.w4_encode(w)), _run(s, x, 2)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    packed = pwlq.w4_encode(w, stream=stream)
    got = pwlq.w4_linear(x, packed, stream=stream), _run(s, x, 2, stream=stream)
    values = pwlq.w4_decode(packed, stream=stream)
    stream.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert torch.equal(values, pwlq.w4_decode(packed))
