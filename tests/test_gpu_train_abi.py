"""The C entries of the training operators, called as a C program calls them."""
import pytest
import torch

from test_train_abi import BLOCK_ARGS, BLOCK_GRADS, FIELDS

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a CUDA device")]

GRADS = "dh lddh dr lddr dx lddx df lddf dpre dpost dgate ws bytes".split()


def _pack(struct, names, floats, **kw):
    v = {k: 0.0 if k in floats else 0 for k in names}
    v.update((k, t.data_ptr() if torch.is_tensor(t) else t) for k, t in kw.items())
    return struct.pack(*(v[k] for k in names))


def block(**kw):
    return _pack(BLOCK_ARGS, FIELDS, ("scale", "eps", "offset", "ratio"), **kw)


def gradients(**kw):
    return _pack(BLOCK_GRADS, GRADS, (), **kw)


def _stream():
    return torch.cuda.current_stream().cuda_stream


def test_the_gradient_of_no_gates_is_not_written():
    from paper_2002_00104_b200 import pwlq
    lib = pwlq.load_library()
    w = torch.ones(64, device="cuda")
    dpre, dpost, dgate = (torch.full((64,), 3.0, device="cuda") for _ in range(3))
    ws = torch.empty(1024, dtype=torch.uint8, device="cuda")
    args = block(rows=0, cols=64, pre=w, post=w, gate=w, ldgate=64, gate_rows=0, gate_tokens=1, scale=1.0, group=64,
                 ratio=0.5, ldc=64)
    assert lib.pwlq_block_norm_backward(args, gradients(lddh=64, lddr=64, lddx=64, lddf=64, dpre=dpre, dpost=dpost,
                                                        dgate=dgate, ws=ws, bytes=1024), _stream()) == pwlq.OK
    assert (dpre == 0).all() and (dpost == 0).all() and (dgate == 3).all()


@pytest.mark.parametrize("rows", [1, 2, 3, 4, 5, 300, 5000])
@pytest.mark.parametrize("tokens", [2 ** 63 - 1, 2 ** 63 - 2, 2 ** 62, 2 ** 31, 2 ** 32 + 1])
@pytest.mark.parametrize("cols", [64, 1200])
def test_gates_of_more_rows_than_there_are(rows, tokens, cols):
    """As if the gate were for exactly the rows; the rows around the gate's gradient stay as they are."""
    from paper_2002_00104_b200 import pwlq
    g = torch.Generator(device="cuda")
    g.manual_seed(rows)
    x, f, dh, dr = (torch.randn(rows, cols, generator=g, device="cuda") for _ in range(4))
    pre, post = (torch.rand(cols, generator=g, device="cuda") + 0.5 for _ in range(2))
    gate = torch.rand(2, cols, generator=g, device="cuda")
    want = pwlq.block_norm(x, f, pre, post, gate, gate_tokens=rows, save=(64, 0.5))
    grads = pwlq.block_norm_backward(want[2], dh, dr)
    got = pwlq.block_norm(x, f, pre, post, gate, gate_tokens=tokens, save=(64, 0.5))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    again = pwlq.block_norm_backward(got[2], dh, dr)
    for k in grads:
        assert torch.equal(grads[k], again[k]), k
    assert (again["dgate"][1] == 0).all()

    lib, saved = pwlq.load_library(), got[2]
    around = torch.full((4, cols), 7.0, device="cuda")
    ws = torch.empty(lib.pwlq_block_norm_backward_workspace_bytes(rows, cols, 2), dtype=torch.uint8, device="cuda")
    args = block(rows=rows, cols=cols, pre=pre, post=post, gate=gate, ldgate=cols, gate_rows=2, gate_tokens=tokens,
                 scale=1.0, eps=1e-6, group=64, ratio=0.5, ldc=saved.r.codes.shape[1], r_codes=saved.r.codes,
                 r_ranges=saved.r.ranges, r_rstd=saved.r_rstd, f_codes=saved.f.codes, f_ranges=saved.f.ranges,
                 f_rstd=saved.f_rstd)
    out = gradients(dh=dh, lddh=cols, dr=dr, lddr=cols, dgate=around[1:], ws=ws, bytes=ws.numel())
    assert lib.pwlq_block_norm_backward(args, out, _stream()) == pwlq.OK
    assert torch.equal(around[1:3], grads["dgate"])
    assert (around[0] == 7).all() and (around[3] == 7).all()


def test_calls_of_different_widths_from_several_threads():
    """Threads that share a kernel, whose calls need 24 to 192 KB of shared memory: every call is accepted
    and gives what it gives alone."""
    import threading

    from paper_2002_00104_b200 import pwlq
    lib, rows = pwlq.load_library(), 4
    cases = []
    for cols in (2048, 8192, 4096, 6144, 16384, 9000):
        g = torch.Generator(device="cuda")
        g.manual_seed(cols)
        x, dh, dr = (torch.randn(rows, cols, generator=g, device="cuda").bfloat16() for _ in range(3))
        pre = torch.ones(cols, device="cuda").bfloat16()
        _, _, saved = pwlq.block_norm(x, None, pre, save=(64, 0.5))
        want = pwlq.block_norm_backward(saved, dh, dr)["dx"]
        dx = torch.empty_like(x)
        args = block(rows=rows, cols=cols, dtype=1, wtype=1, pre=pre, scale=1.0, eps=1e-6, group=64, ratio=0.5,
                     ldc=saved.r.codes.shape[1], r_codes=saved.r.codes, r_ranges=saved.r.ranges, r_rstd=saved.r_rstd)
        out = gradients(dh=dh, lddh=cols, dr=dr, lddr=cols, dx=dx, lddx=cols)
        cases.append((args, out, dx, want, (saved, dh, dr, pre)))
    torch.cuda.synchronize()
    failed = []

    def work(args, out, stream):
        for _ in range(3000):
            if lib.pwlq_block_norm_backward(args, out, stream.cuda_stream) != pwlq.OK:
                failed.append(1)

    threads = [threading.Thread(target=work, args=(*c[:2], torch.cuda.Stream())) for c in cases]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not failed, f"{len(failed)} calls refused"
    for _, _, dx, want, _ in cases:
        assert torch.equal(dx, want)
    assert pwlq.device_status() == 0


@pytest.mark.parametrize("rows,cols", [(1000, 48), (5000, 256), (700, 1040), (3000, 1283), (900, 4104), (300, 8192),
                                       (200, 8704), (200, 8399), (3, 4096)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("norms", ["both", "inner", "outer"])
def test_gradients_written_over_the_gradients_they_come_from(rows, cols, dtype, norms):
    """dx in dr's place and df in dh's, in every form: the bits that separate results have."""
    from paper_2002_00104_b200 import pwlq
    lib, code = pwlq.load_library(), 1 if dtype == torch.bfloat16 else 0
    g = torch.Generator(device="cuda")
    g.manual_seed(rows)
    x, f, dh, dr = (torch.randn(rows, cols, generator=g, device="cuda").to(dtype) for _ in range(4))
    w, gate = torch.ones(cols, device="cuda").to(dtype), torch.rand(2, cols, generator=g, device="cuda").to(dtype)
    pre, post = (w if norms != "inner" else None), (w if norms != "outer" else None)
    _, _, saved = pwlq.block_norm(x, f, pre, post, gate, save=(64, 0.5))
    want = pwlq.block_norm_backward(saved, dh if pre is not None else None, dr)
    some = {"f_codes": saved.f.codes, "f_ranges": saved.f.ranges, "f_rstd": saved.f_rstd if post is not None else 0}
    if pre is not None:
        some.update(r_codes=saved.r.codes, r_ranges=saved.r.ranges, r_rstd=saved.r_rstd)
    args = block(rows=rows, cols=cols, dtype=code, wtype=code, f=f, pre=0 if pre is None else pre,
                 post=0 if post is None else post, gate=gate, ldgate=cols, gate_rows=2, gate_tokens=-(-rows // 2),
                 scale=1.0, eps=1e-6, group=64, ratio=0.5, ldc=saved.f.codes.shape[1], **some)
    dx, df = dr.clone(), dh.clone()
    dgate = torch.empty_like(gate)
    ws = torch.empty(lib.pwlq_block_norm_backward_workspace_bytes(rows, cols, 2), dtype=torch.uint8, device="cuda")
    out = gradients(dh=df if pre is not None else 0, lddh=cols, dr=dx, lddr=cols, dx=dx, lddx=cols, df=df, lddf=cols,
                    dgate=dgate, ws=ws, bytes=ws.numel())
    assert lib.pwlq_block_norm_backward(args, out, _stream()) == pwlq.OK
    for got, name in ((dx, "dx"), (df, "df"), (dgate, "dgate")):
        assert torch.equal(got, want[name]), name
    assert pwlq.device_status() == 0
