"""Arguments of the Python training calls that are refused before any CUDA call."""
import pytest
import torch


@pytest.fixture(scope="module")
def pwlq():
    from paper_2002_00104_b200 import build, pwlq
    build.build()
    pwlq.load_library()
    return pwlq


@pytest.mark.parametrize("group", [2 ** 32 + 64, 2 ** 32 + 32, 2 ** 33 + 256, -2 ** 32 + 128, 257, 0, -64])
def test_group_lengths_beyond_32_bits(pwlq, group):
    """The low 32 bits of some of these are a valid group: taken for it, the call would write more ranges
    than the memory holds.  Refused before the device of the tensors is looked at."""
    x = torch.zeros(4, 512)
    codes = torch.zeros(4, 512, dtype=torch.uint8)
    calls = pwlq._calls()
    for call in (lambda: calls.encode(x, group, 0.5, 0, 0, 0, 0),
                 lambda: calls.decode(codes, 0, 512, 0, 4, 512, group, 0.5, 0, None),
                 lambda: calls.weight_grad(x, codes, 0, 512, 0, 4, 512, group, 0.5, -1, None, 0, None)):
        with pytest.raises(pwlq.PwlqError) as e:
            call()
        assert e.value.status == pwlq.ERR_INVALID_ARG


@pytest.mark.parametrize("cols,group", [(64, 0), (64, -32), (0, 64), (-1, 64)])
def test_checkpoints_of_no_columns_or_groups(pwlq, cols, group):
    codes, ranges = torch.zeros(4, 64, dtype=torch.uint8), torch.zeros(4, 1)
    for make in (lambda: pwlq.Act8(codes, ranges, cols, group, 0.5),
                 lambda: pwlq.act8_empty(4, cols, group, 0.5, "cpu")):
        with pytest.raises(pwlq.PwlqError) as e:
            make()
        assert e.value.status == pwlq.ERR_INVALID_ARG


@pytest.mark.parametrize("failure", ["no compiler", "no headers", "no torch"])
def test_the_library_is_built_where_the_module_of_the_calls_cannot_be(monkeypatch, tmp_path, failure):
    from paper_2002_00104_b200 import build
    built, old = [], tmp_path / "_pwlq_calls.so"
    old.write_bytes(b"of older sources")
    monkeypatch.setattr(build, "CALLS_LIB", str(old))
    monkeypatch.setattr(build, "_nvcc", lambda sources, lib, verbose: built.append(lib))

    def calls(verbose):
        raise {"no compiler": FileNotFoundError("g++"), "no headers": RuntimeError("Python.h: No such file"),
               "no torch": ImportError("No module named 'torch'")}[failure]

    monkeypatch.setattr(build, "_calls", calls)
    with pytest.warns(UserWarning, match="training calls was not built"):
        assert build.build(force=True) == build.LIB
    assert built == [build.LIB, build.PEAK_LIB]
    assert not old.exists()


def test_the_gradient_of_a_block_that_was_not_there(pwlq):
    """df without f: refused before any CUDA call (it was filled with the gradient of r)."""
    from test_train_abi import A, B, BLOCK_GRADS, C, _block
    args = _block(f=0, post=0, gate=0, f_codes=0, f_ranges=0, f_rstd=0)
    grads = BLOCK_GRADS.pack(A, 100, B, 100, A, 100, B, 100, C, 0, 0, 0, 0)
    assert pwlq.load_library().pwlq_block_norm_backward(args, grads, None) == pwlq.ERR_INVALID_ARG


def test_a_checkpoint_without_its_memory(pwlq):
    memory, layout = pwlq.act8_empty(4, 64, device="cpu").detached()
    with pytest.raises(ValueError, match="detached"):
        pwlq.act8_decode(layout)
    assert layout.attached(memory).codes.shape == (4, 64)


@pytest.mark.parametrize("field,value", [("group", 32), ("group", 0), ("rows", 5), ("cols", 600)])
def test_checkpoints_whose_fields_were_changed(pwlq, field, value):
    """More bytes or ranges than the memory holds would be read."""
    saved = pwlq.act8_empty(4, 512, 128, device="cpu")
    setattr(saved, field, value)
    with pytest.raises(ValueError, match="does not hold"):
        pwlq.act8_decode(saved)
