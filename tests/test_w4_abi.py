"""Arguments of the operators on 4-bit weights are checked on the host, before any CUDA call."""
import os
import shutil
import struct
import subprocess

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
W4 = struct.Struct("6q Q")                       # pwlq_w4 and pwlq_w4_moe_args of include/pwlq.h
MOE = struct.Struct("5q Qq Qq QQ Qq QQ Qq")
A, B, C = (0x10000 * i for i in (1, 2, 3))


@pytest.fixture(scope="module")
def pwlq():
    from paper_2002_00104_b200 import build, pwlq
    build.build()
    pwlq.load_library()
    return pwlq


def _w4(**kw):
    v = dict(matrices=1, rows=32, cols=100, group=64, breakpoint=32, paired=0, data=A)
    v.update(kw)
    return W4.pack(*v.values())


def test_structures_have_the_header_s_size(tmp_path):
    cc = shutil.which("gcc") or pytest.skip("no C compiler")
    src = tmp_path / "size.c"
    src.write_text('#include "pwlq.h"\n#include <stdio.h>\nint main(void) { printf("%zu %zu", sizeof(pwlq_w4), '
                   'sizeof(pwlq_w4_moe_args)); return 0; }\n')
    exe = str(tmp_path / "size")
    subprocess.run([cc, "-I", os.path.join(ROOT, "include"), str(src), "-o", exe], check=True)
    sizes = subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split()
    assert [int(v) for v in sizes] == [W4.size, MOE.size]


def test_sizes(pwlq):
    lib = pwlq.load_library()
    assert lib.pwlq_w4_bytes(1, 16, 128, 128, 0) == 1024 + 32
    assert lib.pwlq_w4_bytes(1, 16, 128, 32, 0) == 1024 + 128
    assert lib.pwlq_w4_bytes(3, 17, 129, 64, 0) == 3 * 2 * 2 * (1024 + 64)
    assert lib.pwlq_w4_bytes(1, 18, 1, 256, 1) == 2 * (1024 + 32)         # nine gate rows: two tiles
    for bad in ((0, 16, 128, 128, 0), (1, 0, 128, 128, 0), (1, 16, 0, 128, 0), (1, 16, 128, 16, 0), (1, 17, 128, 128, 1),
                (1, 16, 128, 128, 2), (65536, 16, 128, 128, 0), (1, (1 << 24) + 1, 128, 128, 0),
                (1, 16, (1 << 20) + 1, 128, 0), (65535, 1 << 20, 1 << 20, 128, 0), (1, 16, 128, 2 ** 32 + 64, 0)):
        assert lib.pwlq_w4_bytes(*bad) == 0, bad
    assert pwlq.w4_bytes((3, 17, 129), 64) == 3 * 2 * 2 * (1024 + 64)
    assert lib.pwlq_w4_moe_workspace_bytes(64, 32, 500, 1000) >= 64 * 32 * (1024 * 6 + 8) + 64 * 512 * 6
    for bad in ((65, 2, 100, 100), (1, 33, 100, 100), (1, 0, 100, 100), (-1, 2, 100, 100), (1, 2, 0, 100), (1, 2, 100, 0),
                (1, 2, 100, 2 ** 32)):
        assert lib.pwlq_w4_moe_workspace_bytes(*bad) == 0, bad


@pytest.mark.parametrize("call", ["encode", "decode"])
def test_encode_and_decode(pwlq, call):
    fn = getattr(pwlq.load_library(), "pwlq_w4_" + call)
    good = [_w4(), B, pwlq.F32, 100, 0, None]
    for i, v in ((0, None), (0, _w4(matrices=0)), (0, _w4(rows=0)), (0, _w4(cols=-1)), (0, _w4(group=48)),
                 (0, _w4(breakpoint=0)), (0, _w4(breakpoint=65)), (0, _w4(paired=2)), (0, _w4(rows=33, paired=1)),
                 (0, _w4(data=0)), (0, _w4(data=A + 8)), (1, None), (1, B + 2), (2, 3), (3, 99)):
        args = list(good)
        args[i] = v
        assert fn(*args) == pwlq.ERR_INVALID_ARG, (i, v)
    assert fn(_w4(matrices=2), B, pwlq.F32, 100, -1, None) == pwlq.ERR_INVALID_ARG
    assert fn(_w4(cols=(1 << 20) + 1), B, pwlq.F32, 1 << 21, 0, None) == pwlq.ERR_UNSUPPORTED


def test_linear(pwlq):
    lib = pwlq.load_library()
    size, large = lib.pwlq_w4_linear_workspace_bytes, 16 * 4096
    need = size(4, large, 100, pwlq.BF16, 1)
    assert need == size(4, large, 104, pwlq.BF16, 0) == 4 * 128 * 2
    assert size(3, large, 128, pwlq.F32, 1) == 2304
    assert size(4, large, 104, pwlq.BF16, 1) == size((1 << 19) + 1, large, 100, pwlq.F32, 0) == size(4, large - 16, 100, pwlq.F32, 0) == 0
    for bad in ((0, large, 100, 0, 0), (4, large, 0, 0, 0), (4, large, 100, 3, 0), (-1, large, 100, 0, 0), (4, 0, 100, 0, 0),
                (4, large, 2 ** 32 + 100, 0, 0), (4, -large, 100, 0, 0)):
        assert size(*bad) == 0, bad
    good = [_w4(), B, pwlq.BF16, 4, 100, C, 32, 0x50000, need, None]
    big = [_w4(rows=large), B, pwlq.BF16, 4, 100, 0x10000000, large, 0x50000, need, None]

    def rc(*changes):
        args = list(good)
        for i, v in changes:
            args[i] = v
        return lib.pwlq_w4_linear(*args)

    for i, v in ((0, None), (0, _w4(matrices=2)), (1, None), (1, B + 1), (2, 7), (3, -1), (4, 99), (5, None), (5, C + 1),
                 (6, 31), (5, B), (5, B + 2 * 99), (5, B - 2)):
        assert rc((i, v)) == pwlq.ERR_INVALID_ARG, (i, v)
    assert rc((3, (1 << 19) + 1)) == pwlq.ERR_UNSUPPORTED
    for i, v, status in ((7, None, pwlq.ERR_WORKSPACE), (8, need - 1, pwlq.ERR_WORKSPACE), (7, 0x50000 + 128, pwlq.ERR_INVALID_ARG)):
        args = list(big)
        args[i] = v
        assert lib.pwlq_w4_linear(*args) == status
    assert rc((3, 0), (1, None), (5, None)) == pwlq.OK
    # columns of the same rows: beside each other they are no overlap, but the call would launch; off by one they are
    assert rc((4, 200), (6, 200), (5, B + 2 * 99)) == pwlq.ERR_INVALID_ARG
    assert rc((4, 200), (6, 200), (5, B + 2 * 169)) == pwlq.ERR_INVALID_ARG


def test_moe(pwlq):
    import ctypes
    lib = pwlq.load_library()
    need = lib.pwlq_w4_moe_workspace_bytes(4, 2, 100, 24)
    keep = []

    def block(**kw):
        v = dict(tokens=4, top=2, dtype=pwlq.BF16, router_dtype=pwlq.F32, normalize=1, x=A, ldx=100, router=B, ldrouter=100,
                 up=dict(), down=dict(), y=C, ldy=100, chosen=0, weights=0, workspace=A, bytes=need)
        v.update(kw)
        for name, default in (("up", dict(matrices=8, rows=48, cols=100, paired=1)),
                              ("down", dict(matrices=8, rows=100, cols=24, paired=0))):
            if isinstance(v[name], dict):
                b = ctypes.create_string_buffer(_w4(**{**default, **v[name]}))
                keep.append(b)
                v[name] = ctypes.addressof(b)
        return MOE.pack(*v.values())

    def rc(**kw):
        return lib.pwlq_w4_moe(block(**kw), None)

    assert lib.pwlq_w4_moe(None, None) == pwlq.ERR_INVALID_ARG
    for bad in (dict(tokens=-1), dict(top=0), dict(top=9), dict(dtype=5), dict(router_dtype=pwlq.F16), dict(normalize=2),
                dict(x=0), dict(x=A + 1), dict(ldx=99), dict(router=0), dict(router=B + 2), dict(ldrouter=99), dict(up=0),
                dict(down=0), dict(up=dict(paired=0)), dict(down=dict(paired=1)), dict(up=dict(matrices=7)),
                dict(up=dict(cols=99)), dict(down=dict(cols=25)), dict(y=0), dict(y=C + 1), dict(ldy=99),
                dict(chosen=A + 2), dict(weights=A + 1), dict(workspace=A + 128), dict(up=dict(data=0))):
        assert rc(**bad) == pwlq.ERR_INVALID_ARG, bad
    assert rc(tokens=65, bytes=1 << 40) == pwlq.ERR_UNSUPPORTED
    assert rc(top=33, up=dict(matrices=64), down=dict(matrices=64)) == pwlq.ERR_UNSUPPORTED
    assert rc(up=dict(matrices=1025), down=dict(matrices=1025)) == pwlq.ERR_UNSUPPORTED
    assert rc(workspace=0) == rc(bytes=need - 1) == rc(bytes=-1) == pwlq.ERR_WORKSPACE
    assert rc(tokens=0, x=0, y=0, workspace=0) == pwlq.OK


@pytest.mark.parametrize("group", [0, -32, 16, 48, 2 ** 32 + 64])
def test_groups(pwlq, group):
    x = torch.zeros(16, 128)
    for call in (lambda: pwlq.w4_bytes((16, 128), group), lambda: pwlq.w4_encode(x, group=group),
                 lambda: pwlq.W4(torch.zeros(1056, dtype=torch.uint8), (16, 128), group)):
        with pytest.raises(pwlq.PwlqError) as e:
            call()
        assert e.value.status == pwlq.ERR_INVALID_ARG


@pytest.mark.parametrize("ratio", [0.0, 1.5, 0.3, -0.5, float("nan"), 1 / 128, float("inf")])
def test_ratios(pwlq, ratio):
    with pytest.raises(pwlq.PwlqError):
        pwlq.w4_encode(torch.zeros(16, 128), ratio=ratio)


def test_shapes_and_memory(pwlq):
    for shape in ((128,), (0, 128), (16, 0), (2, 2, 16, 128), (-1, 128)):
        with pytest.raises((ValueError, pwlq.PwlqError)):
            pwlq.w4_bytes(shape)
    with pytest.raises(pwlq.PwlqError):
        pwlq.w4_bytes((17, 128), paired=True)
    good = torch.zeros(1056, dtype=torch.uint8)
    packed = pwlq.W4(good, (16, 128), 128, 0.25)
    assert (packed.shape, packed.group, packed.ratio, packed.paired) == ((16, 128), 128, 0.25, False)
    for memory in (good[:1055], torch.zeros(1056), torch.zeros(2112, dtype=torch.uint8)[::2]):
        with pytest.raises(ValueError, match="1056"):
            pwlq.W4(memory, (16, 128), 128, 0.25)
    for name in ("shape", "group", "ratio", "paired", "memory"):     # what the calls trust cannot be changed
        with pytest.raises(AttributeError):
            setattr(packed, name, 1)


def test_sizes_beyond_the_limits(pwlq):
    for shape in ((65536, 16, 128), (1, (1 << 24) + 1, 128), (16, (1 << 20) + 1), (65535, 1 << 20, 1 << 20)):
        with pytest.raises(pwlq.PwlqError) as e:
            pwlq.w4_bytes(shape)
        assert e.value.status == pwlq.ERR_UNSUPPORTED
    wide = torch.zeros(1, dtype=torch.bfloat16).expand(16, (1 << 20) + 1)
    with pytest.raises(pwlq.PwlqError) as e:
        pwlq.w4_encode(wide)
    assert e.value.status == pwlq.ERR_UNSUPPORTED


def test_tensors_that_are_not_on_the_device(pwlq):
    x = torch.zeros(16, 128)
    packed = pwlq.W4(torch.zeros(1056, dtype=torch.uint8), (16, 128))
    pair = pwlq.W4(torch.zeros(2 * 1056, dtype=torch.uint8), (1, 32, 128), paired=True)
    down = pwlq.W4(torch.zeros(8 * 1056, dtype=torch.uint8), (1, 128, 16))
    for bad in (lambda: pwlq.w4_encode(x), lambda: pwlq.w4_encode(None), lambda: pwlq.w4_decode(packed),
                lambda: pwlq.w4_linear(x, packed), lambda: pwlq.w4_linear(None, packed),
                lambda: pwlq.w4_moe(x, x[:1], pair, down, 1)):
        with pytest.raises((ValueError, AttributeError)):
            bad()
