"""The binding's look at its tensors: the native module is of this interpreter and this torch, and what
stands in for it where there is none answers alike."""
import sys
import sysconfig

import pytest


@pytest.fixture
def both(monkeypatch):
    """The native functions, and the ones that the binding uses without the module."""
    import paper_2607_23815_amd as package
    from paper_2607_23815_amd import _tensor_address as native, lib
    monkeypatch.setattr(lib, "_address", None)
    monkeypatch.setattr(lib, "_rows_address", None)
    lib._find_address()
    assert (lib._address, lib._rows_address) == (native.address, native.rows_address)
    monkeypatch.delattr(package, "_tensor_address")
    monkeypatch.setitem(sys.modules, "paper_2607_23815_amd._tensor_address", None)
    lib._find_address()
    assert lib._address is not native.address and lib._rows_address is not native.rows_address
    return native, lib


def same(native, lib, tensors, dtypes, shapes, dev):
    for x in tensors:
        for dtype in dtypes:
            for d in (dev, dev + 1):
                assert lib._address(x, dtype, d) == native.address(x, dtype, d)
                for s in shapes:
                    assert lib._rows_address(x, dtype, d, *s) == native.rows_address(x, dtype, d, *s)


def test_the_module_is_of_this_interpreter_and_torch():
    import torch
    from paper_2607_23815_amd import _tensor_address as native
    assert native.__file__.endswith(sysconfig.get_config_var("EXT_SUFFIX"))
    assert native.torch_version == torch.__version__


def test_a_module_of_another_torch_is_not_used(monkeypatch):
    from paper_2607_23815_amd import _tensor_address as native, lib
    monkeypatch.setattr(native, "torch_version", "1.0")
    monkeypatch.setattr(lib, "_address", None)
    monkeypatch.setattr(lib, "_rows_address", None)
    lib._find_address()
    assert lib._address is not native.address and lib._rows_address is not native.rows_address


def test_host_tensors(both):
    import torch
    native, lib = both
    t = torch.zeros((2, 3, 4), dtype=torch.bfloat16)
    same(native, lib, (t, t.to_sparse(), None, 3, t.to("meta")), (torch.bfloat16, torch.int32),
         [(2, 3, 4)], 0)
    assert lib._address(t, torch.bfloat16, 0) is None


@pytest.mark.gpu
def test_gpu_tensors(gpu_lib, both):
    import torch
    native, lib = both
    bf, dev = torch.bfloat16, torch.cuda.current_device()
    t = torch.zeros((2, 3, 4), dtype=bf, device="cuda")
    wide = torch.zeros((5, 9, 4), dtype=bf, device="cuda")
    tensors = (t, t[:1], t[:, :1], t[:0], t.transpose(0, 1), wide[:2, 2:5], wide[::2, 4:5], wide[..., ::2],
               wide[:1, 3:6], t.int(), t.cpu(), t.to_sparse(), t[0], None)
    shapes = [(2, 3, 4), (1, 3, 4), (2, 1, 4), (3, 1, 4), (0, 3, 4), (3, 2, 4), (5, 9, 2)]
    same(native, lib, tensors, (bf, torch.int32, torch.float32), shapes, dev)
    assert lib._address(t, bf, dev) == t.data_ptr()
    assert lib._rows_address(wide[:2, 2:5], bf, dev, 2, 3, 4) == (wide.data_ptr() + 2 * 4 * 2, 36)


@pytest.mark.gpu
def test_a_step_without_the_module(gpu_lib, both):
    """The calls run, and refuse, as with it."""
    from tests import test_gpu_sparse_step as step
    step.test_sparse_rows_of_a_decode_step_without_row_seq(gpu_lib)
    step.test_the_binding_refuses_wrong_tensors(gpu_lib)
