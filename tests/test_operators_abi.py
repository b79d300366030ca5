"""CPU tier: the calls around sparse reads of the cache refuse bad arguments on the host, before
any launch, and take empty calls as successful no-ops (no GPU is touched here)."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def lib():
    from paper_2607_23815_amd import lib as L
    return L


FAKE = ctypes.c_void_p(0x3000)  # (host-side checks never dereference an address)


def refused(lib, status, got, *words):
    assert got == status, lib.pkv_last_error()
    for w in words:
        assert w in lib.pkv_last_error(), lib.pkv_last_error()


def _extend(lib, **kw):
    a = dict(tables=FAKE, max_blocks=4, cached=FAKE, new=FAKE, num_seqs=2, free=FAKE, num_free=3,
             used=FAKE, used_out=FAKE, cu=FAKE, lens=FAKE, status=FAKE, max_rows=8, slots=None,
             row_seq=None, positions=None, row_lens=None)
    a.update(kw)
    return lib._lib.pkv_extend_tables(*a.values(), None)


@pytest.mark.parametrize("bad", [
    dict(tables=None), dict(cached=None), dict(new=None), dict(free=None), dict(used=None),
    dict(used_out=None), dict(cu=None), dict(lens=None), dict(status=None), dict(max_blocks=-1),
    dict(num_seqs=-1), dict(num_free=-1), dict(max_rows=-1), dict(max_rows=2**30 + 1)])
def test_extend_tables_refuses(lib, bad):
    refused(lib, lib.PKV_ERR_INVALID_ARG, _extend(lib, **bad), "pkv_extend_tables")


def test_binding_refuses_host_tensors(lib):
    import torch
    if torch.cuda.is_available():
        pytest.skip("for a box without a GPU")
    with pytest.raises((TypeError, RuntimeError, AssertionError)):
        z = torch.zeros(1, dtype=torch.int32)
        lib.pkv_extend_tables(z.view(1, 1), z, z, z, z, z, torch.zeros(2, dtype=torch.int32), z, z,
                              0)
