"""Calls on 4-bit weights as a host program makes them: from several threads at once through the C ABI."""
import ctypes
import struct
import threading

import pytest
import torch

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a CUDA device")]

W4 = struct.Struct("6q Q")                       # pwlq_w4 and pwlq_w4_moe_args of include/pwlq.h
MOE = struct.Struct("5q Qq Qq QQ Qq QQ Qq")


def _weights(seed, *shape):
    g = torch.Generator("cuda").manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * shape[-1] ** -0.5).bfloat16()


class _Layer:
    """A call of pwlq_w4_moe with memory of its own."""

    def __init__(self, seed, tokens, experts, features, hidden, top):
        from paper_2002_00104_b200 import pwlq
        self.lib, self.stream = pwlq.load_library(), torch.cuda.Stream()
        up = pwlq.w4_encode(_weights(seed, experts, 2 * hidden, features), group=64, paired=True)
        down = pwlq.w4_encode(_weights(seed + 1, experts, features, hidden), group=64)
        router, x = _weights(seed + 2, experts, features), _weights(seed + 3, tokens, features)
        self.want = pwlq.w4_moe(x, router, up, down, top)
        self.y = torch.zeros_like(x)
        need = pwlq.w4_moe_workspace_bytes(tokens, top, features, hidden)
        workspace = torch.zeros(need, dtype=torch.uint8, device="cuda")
        blocks = [ctypes.create_string_buffer(W4.pack(*p._fields, p.memory.data_ptr())) for p in (up, down)]
        self.keep = up, down, router, x, workspace, blocks
        self.args = MOE.pack(tokens, top, pwlq.BF16, pwlq.BF16, 1, x.data_ptr(), features, router.data_ptr(), features,
                             *(ctypes.addressof(b) for b in blocks), self.y.data_ptr(), features, 0, 0,
                             workspace.data_ptr(), need)

    def call(self):
        return self.lib.pwlq_w4_moe(self.args, self.stream.cuda_stream)


def test_layers_of_different_sizes_from_several_threads():
    """The same kernels with different amounts of shared memory: no thread's launch depends on what another's asks for."""
    layers = [_Layer(1, 1, 64, 48, 64, 4), _Layer(11, 64, 64, 48, 64, 4), _Layer(21, 9, 1024, 48, 64, 4)]
    torch.cuda.synchronize()
    failed = [0] * len(layers)

    def work(i):
        torch.cuda.set_device(0)
        for n in range(1500):
            failed[i] += layers[i].call() != 0
            if n % 100 == 99:
                layers[i].stream.synchronize()

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(layers))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert failed == [0] * len(layers)
    for v in layers:
        assert torch.equal(v.y, v.want)


def test_decoding_to_matrices_whose_rows_lie_between_one_another_s():
    from paper_2002_00104_b200 import pwlq
    packed = pwlq.w4_encode(_weights(31, 3, 40, 200), group=64)
    want = pwlq.w4_decode(packed)
    for gap in (0, 5):
        out = torch.full((40, 3, 200 + gap), 7.0, device="cuda")
        view = out.transpose(0, 1)[..., :200]
        pwlq.w4_decode(packed, out=view)
        assert torch.equal(view, want) and (out[..., 200:] == 7).all()
    flat = torch.zeros(40 * 600, device="cuda")
    for strides in ((199, 600, 1), (100, 200, 1), (200, 500, 1), (0, 200, 1)):
        with pytest.raises(ValueError):
            pwlq.w4_decode(packed, out=flat.as_strided((3, 40, 200), strides))


def test_what_a_layer_refuses_and_as_what():
    """The C entry's status for each, whoever finds it."""
    from paper_2002_00104_b200 import pwlq
    experts, features, hidden = 40, 128, 64
    up = pwlq.w4_encode(_weights(41, experts, 2 * hidden, features), group=64, paired=True)
    down = pwlq.w4_encode(_weights(42, experts, features, hidden), group=64)
    router, x = _weights(43, experts, features), _weights(44, 4, features)
    few = [pwlq.w4_encode(pwlq.w4_decode(v)[:8], group=64, paired=v.paired) for v in (up, down)]
    workspace = torch.zeros(pwlq.w4_moe_workspace_bytes(4, 2, features, hidden), dtype=torch.uint8, device="cuda")
    unpaired = pwlq.w4_encode(_weights(45, experts, 2 * hidden, features), group=64)
    many = pwlq.w4_encode(_weights(46, 1, 32, 32).expand(1025, 32, 32), group=32, paired=True)
    for status, args, kw in (
            (pwlq.ERR_INVALID_ARG, (x, router, up, down, 0), {}), (pwlq.ERR_INVALID_ARG, (x, router, up, down, -1), {}),
            (pwlq.ERR_INVALID_ARG, (x, router[:8], *few, 9), {}), (pwlq.ERR_INVALID_ARG, (x, router[:8], *few, 33), {}),
            (pwlq.ERR_INVALID_ARG, (x, router, up, down, 41), {}), (pwlq.ERR_INVALID_ARG, (x, router, up, down, 2 ** 32 + 2), {}),
            (pwlq.ERR_UNSUPPORTED, (x, router, up, down, 33), {}), (pwlq.ERR_UNSUPPORTED, (x[:1].repeat(65, 1), router, up, down, 2), {}),
            (pwlq.ERR_INVALID_ARG, (x, router, up, up, 2), {}), (pwlq.ERR_INVALID_ARG, (x, router, unpaired, down, 2), {}),
            (pwlq.ERR_INVALID_ARG, (x, router, up, few[1], 2), {}),
            (pwlq.ERR_UNSUPPORTED, (x[:, :32], _weights(47, 1025, 32), many, pwlq.w4_encode(_weights(48, 1, 32, 16).expand(1025, 32, 16), group=32), 2), {}),
            (pwlq.ERR_WORKSPACE, (x, router, up, down, 2), dict(workspace=workspace[:-1])),
            (pwlq.ERR_WORKSPACE, (x, router, up, down, 2), dict(workspace=workspace[:0])),
            (pwlq.ERR_INVALID_ARG, (x, router, up, down, 2), dict(workspace=torch.zeros(workspace.numel() + 8, dtype=torch.uint8, device="cuda")[8:]))):
        with pytest.raises(pwlq.PwlqError) as e:
            pwlq.w4_moe(*args, **kw)
        assert e.value.status == status, (args[4], kw, e.value)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_products_into_the_gaps_of_their_tokens_rows(dtype):
    """x and out in one piece of memory with different pitches: what does not meet is taken, what does is refused."""
    from paper_2002_00104_b200 import pwlq
    packed = pwlq.w4_encode(_weights(51, 16, 40), group=32)
    values = torch.randn(4, 40, generator=torch.Generator("cuda").manual_seed(5), device="cuda").to(dtype)
    want = pwlq.w4_linear(values, packed)
    memory = torch.full((2048,), 7.0, dtype=dtype, device="cuda")
    x = memory.as_strided((4, 40), (100, 1), 0)          # 0-39, 100-139, 200-239, 300-339
    x.copy_(values)
    for at, pitch in ((40, 120), (60, 110), (60, 108), (340, 16), (40, 100)):
        y = memory.as_strided((4, 16), (pitch, 1), at)
        pwlq.w4_linear(x, packed, out=y)
        assert torch.equal(y, want) and torch.equal(x, values), (at, pitch)
        y.fill_(7.0)
    for at, pitch in ((39, 120), (40, 90), (60, 90), (25, 300), (60, 65), (124, 16)):
        with pytest.raises(pwlq.PwlqError) as e:
            pwlq.w4_linear(x, packed, out=memory.as_strided((4, 16), (pitch, 1), at))
        assert e.value.status == pwlq.ERR_INVALID_ARG and torch.equal(x, values)
