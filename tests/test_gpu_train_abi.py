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
