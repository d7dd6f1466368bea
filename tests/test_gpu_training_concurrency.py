"""The training calls in CUDA graphs, on several streams at once and from several threads."""
import threading

import pytest
import torch

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a CUDA device")]


def _inputs(seed, rows=700, cols=1280, outputs=520):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def rand(*shape):
        return torch.randn(*shape, generator=g, device="cuda").bfloat16()

    return {"x": rand(rows, cols), "f": rand(rows, cols), "pre": rand(cols), "post": rand(cols), "gate": rand(3, cols),
            "dh": rand(rows, cols), "dr": rand(rows, cols), "dy": rand(rows, outputs), "odd": rand(rows, 515)}


def _step(s):
    """Every call once; the weight gradients of an aligned dy and of one that is copied first."""
    from paper_2002_00104_b200 import pwlq
    r, h, saved = pwlq.block_norm(s["x"], s["f"], s["pre"], s["post"], s["gate"], save=(64, 0.4375))
    grads = pwlq.block_norm_backward(saved, s["dh"], s["dr"])
    kept = pwlq.act8_encode(h, group=128, ratio=0.5)
    return [r, h, *grads.values(), pwlq.act8_decode(kept, dtype=torch.bfloat16), pwlq.act8_weight_grad(s["dy"], kept),
            pwlq.act8_weight_grad(s["odd"], kept, dtype=torch.float32)]


def test_captured_calls_replayed_on_other_inputs():
    from paper_2002_00104_b200 import pwlq
    s = _inputs(0, rows=2000)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _step(s)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = _step(s)
    for seed in (1, 2):
        for k, v in _inputs(seed, rows=2000).items():
            s[k].copy_(v)
        graph.replay()
        for a, b in zip(out, _step(s)):
            assert torch.equal(a, b)
    assert pwlq.device_status() == 0


@pytest.mark.parametrize("threads", [False, True])
def test_calls_side_by_side(threads):
    """Four streams, each with its own inputs, whose kernels overlap: what every one gives alone."""
    from paper_2002_00104_b200 import pwlq
    inputs = [_inputs(i, rows=300 + 500 * i) for i in range(4)]
    want = [_step(s) for s in inputs]
    streams = [torch.cuda.Stream() for _ in inputs]
    got = [None] * len(inputs)
    torch.cuda.synchronize()

    def work(i, times):
        torch.cuda.set_device(0)
        with torch.cuda.stream(streams[i]):
            for _ in range(times):
                got[i] = _step(inputs[i])

    if threads:
        workers = [threading.Thread(target=work, args=(i, 20)) for i in range(len(inputs))]
        for t in workers:
            t.start()
        for t in workers:
            t.join()
    else:
        for _ in range(20):
            for i in range(len(inputs)):
                work(i, 1)
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        for u, v in zip(a, b):
            assert torch.equal(u, v)
    assert pwlq.device_status() == 0
