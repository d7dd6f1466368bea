"""Pitches that the C entries on 4-bit weights take: checked on the host, before any CUDA call."""
import struct

import pytest

W4 = struct.Struct("6q Q")                       # pwlq_w4 of include/pwlq.h


@pytest.fixture(scope="module")
def pwlq():
    from paper_2002_00104_b200 import build, pwlq
    build.build()
    pwlq.load_library()
    return pwlq


@pytest.mark.parametrize("matrices,rows,cols,ldy,ldm", [
    (2, 32, 100, 100, 0), (2, 32, 100, 100, 99), (2, 32, 100, 100, 3199), (2, 32, 100, 128, 31 * 128 + 99), (2, 1, 100, 100, 99),
    (3, 32, 100, 300, 99), (3, 32, 100, 299, 100), (3, 32, 100, 1000, 451), (3, 32, 100, 300, 450), (2, 1 << 20, 1, 1 << 40, 1 << 40)])
def test_decode_refuses_matrices_that_overlap(pwlq, matrices, rows, cols, ldy, ldm):
    """They would be written side by side, in no order."""
    w = W4.pack(matrices, rows, cols, 64, 32, 0, 0x10000)
    # no GPU is reached with them: what is not refused here would launch
    assert pwlq.load_library().pwlq_w4_decode(w, 0x20000, pwlq.F32, ldy, ldm, None) == pwlq.ERR_INVALID_ARG
