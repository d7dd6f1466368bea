"""Arguments of the training operators are checked on the host, before any CUDA call."""
import os
import struct

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    from paper_2002_00104_b200 import build, pwlq
    build.build()
    return pwlq.load_library()


# pwlq_block_norm_args and pwlq_block_norm_grads of include/pwlq.h
BLOCK_ARGS = struct.Struct("4q QqQqQQQqqq 3d QqQq qdq QQQQQQ")
BLOCK_GRADS = struct.Struct("QqQqQqQq QQQ Qq")

A, B, C = (0x10000 * i for i in (1, 2, 3))


def test_encode_and_decode(lib):
    from paper_2002_00104_b200 import pwlq
    good = [A, pwlq.F32, 4, 100, 100, 64, 0.5, B, 112, C, None]

    def rc(i, v):
        args = list(good)
        args[i] = v
        return lib.pwlq_act8_encode(*args)

    for i, v in ((0, None), (0, A + 2), (1, 3), (2, -1), (3, 0), (4, 99), (5, 16), (6, 0.0), (6, 1.01),
                 (6, float("nan")), (6, 2.0 ** -21), (6, 1 - 2.0 ** -13), (7, None), (7, B + 8), (8, 96), (8, 104), (9, None),
                 (9, C + 2)):
        assert rc(i, v) == pwlq.ERR_INVALID_ARG, (i, v)
    assert rc(2, 1 << 31) == pwlq.ERR_UNSUPPORTED
    assert rc(3, 1 << 25) == pwlq.ERR_UNSUPPORTED
    assert rc(2, 0) == pwlq.OK
    assert lib.pwlq_act8_decode(B, 112, C, 4, 100, 64, 0.5, A + 2, pwlq.F32, 100, None) == pwlq.ERR_INVALID_ARG
    assert lib.pwlq_act8_decode(B, 112, C, 0, 100, 64, 0.5, A, pwlq.F32, 100, None) == pwlq.OK


FIELDS = ("rows cols dtype wtype x ldx f ldf post pre gate ldgate gate_rows gate_tokens scale eps offset r "
          "ldr h ldh group ratio ldc r_codes r_ranges r_rstd f_codes f_ranges f_rstd").split()


def _block(**kw):
    v = dict(rows=4, cols=100, dtype=0, wtype=0, x=A, ldx=100, f=B, ldf=100, post=C, pre=C, gate=A, ldgate=100,
             gate_rows=2, gate_tokens=2, scale=1.0, eps=1e-6, offset=0.0, r=A, ldr=100, h=B, ldh=100, group=64,
             ratio=0.5, ldc=112, r_codes=A, r_ranges=A, r_rstd=A, f_codes=A, f_ranges=A, f_rstd=A)
    v.update(kw)
    return BLOCK_ARGS.pack(*(v[k] for k in FIELDS))


def test_block_norm(lib):
    from paper_2002_00104_b200 import pwlq
    assert lib.pwlq_block_norm(None, None) == pwlq.ERR_INVALID_ARG
    for bad in (dict(cols=0), dict(rows=-1), dict(dtype=7), dict(wtype=1), dict(x=0), dict(x=A + 2),
                dict(ldx=99), dict(f=0), dict(ldf=5), dict(post=C + 1), dict(gate_rows=1), dict(gate_tokens=0),
                dict(ldgate=9), dict(pre=0), dict(h=0), dict(ldh=3), dict(r=A + 1), dict(group=8),
                dict(ratio=0.0), dict(ldc=100), dict(ldc=96), dict(r_codes=A + 4), dict(r_ranges=0),
                dict(f_ranges=A + 2), dict(f_rstd=A + 1), dict(r=0, pre=0, h=0)):
        assert lib.pwlq_block_norm(_block(**bad), None) == pwlq.ERR_INVALID_ARG, bad
    assert lib.pwlq_block_norm(_block(cols=16385, ldx=16385), None) == pwlq.ERR_UNSUPPORTED
    assert lib.pwlq_block_norm(_block(rows=0, gate_rows=0), None) == pwlq.OK


def test_block_norm_backward(lib):
    from paper_2002_00104_b200 import pwlq
    need = lib.pwlq_block_norm_backward_workspace_bytes(4, 100, 2)
    assert need > 0
    assert lib.pwlq_block_norm_backward_workspace_bytes(4, 0, 2) == 0
    assert lib.pwlq_block_norm_backward_workspace_bytes(4, 16385, 2) == 0
    names = "dh lddh dr lddr dx lddx df lddf dpre dpost dgate ws bytes".split()

    def rc(block=None, **kw):
        v = dict(dh=A, lddh=100, dr=B, lddr=100, dx=A, lddx=100, df=B, lddf=100, dpre=C, dpost=C, dgate=C,
                 ws=A, bytes=need)
        v.update(kw)
        return lib.pwlq_block_norm_backward(block or _block(), BLOCK_GRADS.pack(*(v[k] for k in names)),
                                            None)

    assert lib.pwlq_block_norm_backward(_block(), None, None) == pwlq.ERR_INVALID_ARG
    for bad in (dict(dh=0), dict(lddh=99), dict(dr=A + 1), dict(lddx=1), dict(df=B + 2), dict(dpre=C + 1),
                dict(block=_block(pre=0)), dict(block=_block(r_codes=0)), dict(block=_block(r_rstd=0)),
                dict(block=_block(f_codes=0)), dict(block=_block(f_rstd=0)), dict(block=_block(group=1)),
                dict(ws=A + 128), dict(block=_block(gate=0))):
        assert rc(**bad) == pwlq.ERR_INVALID_ARG, bad
    assert rc(bytes=need - 1) == rc(ws=0) == pwlq.ERR_WORKSPACE


def test_weight_grad(lib):
    from paper_2002_00104_b200 import pwlq
    need = lib.pwlq_act8_weight_grad_workspace_bytes(8, 32, 100, 0)
    assert need > 0 and lib.pwlq_act8_weight_grad_workspace_bytes(8, 0, 100, 0) == 0
    good = [A, pwlq.BF16, 8, 32, 33, B, 112, C, 100, 64, 0.5, A, pwlq.F32, 100, 0, A, need, None]

    def rc(i, v):
        args = list(good)
        args[i] = v
        return lib.pwlq_act8_weight_grad(*args)

    for i, v in ((0, None), (0, A + 1), (1, 9), (2, -1), (3, 0), (4, 31), (5, None), (5, B + 1), (6, 100),
                 (7, C + 2), (8, 0), (9, 7), (10, 0.0), (11, None), (11, A + 2), (12, pwlq.F16), (13, 99),
                 (15, A + 16)):
        assert rc(i, v) == pwlq.ERR_INVALID_ARG, (i, v)
    assert rc(1, pwlq.F32) == pwlq.ERR_UNSUPPORTED
    assert rc(16, need - 1) == rc(15, None) == pwlq.ERR_WORKSPACE


def test_the_compiled_calls_refuse_what_is_no_cuda_tensor(lib):
    import torch
    from paper_2002_00104_b200 import pwlq
    x = torch.zeros(4, 64)
    for bad in (lambda: pwlq.act8_encode(x), lambda: pwlq.act8_encode(None),
                lambda: pwlq.block_norm(x, x, pre_weight=x[0]),
                lambda: pwlq.act8_weight_grad(x, pwlq.Act8(torch.zeros(4, 64, dtype=torch.uint8), x, 64, 64, 0.5)),
                lambda: pwlq.act8_decode(pwlq.Act8(torch.zeros(4, 64, dtype=torch.uint8), x, 64, 64, 0.5))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises((TypeError, ValueError)):
        pwlq._calls().encode(x)


def test_packed_blocks_have_the_header_s_size(lib, tmp_path):
    import shutil
    import subprocess
    cc = shutil.which("gcc") or pytest.skip("no C compiler")
    src = tmp_path / "size.c"
    src.write_text('#include "pwlq.h"\n#include <stdio.h>\nint main(void) { printf("%zu %zu", '
                   'sizeof(pwlq_block_norm_args), sizeof(pwlq_block_norm_grads)); return 0; }\n')
    exe = str(tmp_path / "size")
    subprocess.run([cc, "-I", os.path.join(ROOT, "include"), str(src), "-o", exe], check=True)
    sizes = subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split()
    assert [int(v) for v in sizes] == [BLOCK_ARGS.size, BLOCK_GRADS.size]
