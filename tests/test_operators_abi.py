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


def _kv(lib, head_dim=128, block_size=16, hkv=2):
    return lib.PagedKV(0x1000, 0x2000, 10, block_size, hkv, head_dim)


def _rope(lib, kv=None, rope=None, **kw):
    a = dict(q=FAKE, q_stride=512, hq=4, k=FAKE, k_stride=256, v=FAKE, v_stride=256, slots=FAKE,
             positions=FAKE, pos_stride=5, rows=5, q_out=FAKE, q_out_stride=512)
    a.update(kw)
    rope = lib.rope_spec([1.0] * 64, axis_of=[0, 1] * 32) if rope is None else rope
    return lib._lib.pkv_rope_append(ctypes.byref(kv or _kv(lib)),
                                    ctypes.byref(rope) if rope else None, *a.values(), None)


@pytest.mark.parametrize("bad", [
    dict(q=None), dict(k=None), dict(v=None), dict(slots=None), dict(positions=None),
    dict(q_out=None), dict(q=ctypes.c_void_p(0x3008)), dict(k=ctypes.c_void_p(0x3002)),
    dict(v=ctypes.c_void_p(0x3004)), dict(q_out=ctypes.c_void_p(0x3008)), dict(q_stride=504),
    dict(q_stride=516), dict(k_stride=248), dict(v_stride=257), dict(q_out_stride=-512),
    dict(pos_stride=4), dict(rows=-1), dict(rows=2**27)])
def test_rope_append_refuses(lib, bad):
    refused(lib, lib.PKV_ERR_INVALID_ARG, _rope(lib, **bad), "pkv_rope_append")


def test_rope_append_refuses_shapes(lib):
    shape = lib.PKV_ERR_UNSUPPORTED_SHAPE
    refused(lib, shape, _rope(lib, hq=3), "num_q_heads")
    refused(lib, shape, _rope(lib, hq=0), "num_q_heads")
    refused(lib, shape, _rope(lib, kv=_kv(lib, 96)), "head_dim")
    refused(lib, shape, _rope(lib, kv=_kv(lib, 128, 32)), "block_size")
    refused(lib, shape, _rope(lib, rope=lib.rope_spec([1.0] * 9)), "rot_dim")
    refused(lib, shape, _rope(lib, kv=_kv(lib, 64)), "rot_dim")
    arg = lib.PKV_ERR_INVALID_ARG
    refused(lib, arg, _rope(lib, rope=False), "rope is NULL")
    refused(lib, arg, _rope(lib, rope=lib.rope_spec([1.0] * 8, scale=float("nan"))), "scale")
    refused(lib, arg, _rope(lib, rope=lib.rope_spec([float("inf")] * 8)), "inv_freq")
    refused(lib, arg, _rope(lib, rope=lib.rope_spec([1.0] * 8, axis_of=[1] * 8, num_axes=1)),
            "axis_of")
    refused(lib, arg, _rope(lib, rope=lib.rope_spec([1.0] * 8, num_axes=5)), "num_axes")
    refused(lib, arg, lib._lib.pkv_rope_append(None, *[None] * 2, 0, 4, None, 0, None, 0, None,
                                               None, 0, 0, None, 0, None), "kv is NULL")
    assert _rope(lib, rows=0, q=None, k=None, v=None, slots=None) == lib.PKV_OK
    for freqs, axes in (([1.0] * 65, None), ([1.0] * 8, [0] * 7), ([1.0], [4]), ([1.0], [-1])):
        with pytest.raises(ValueError):
            lib.rope_spec(freqs, axis_of=axes)


def _bounds(lib, kv=None, **kw):
    a = dict(bounds=FAKE, tables=FAKE, max_blocks=4, cached=FAKE, cu=FAKE, num_seqs=2, max_new=3)
    a.update(kw)
    return lib._lib.pkv_block_bounds(ctypes.byref(kv or _kv(lib)), *a.values(), None)


def test_block_bounds_refuses(lib):
    for bad in (dict(bounds=None), dict(tables=None), dict(cached=None), dict(cu=None),
                dict(bounds=ctypes.c_void_p(0x3008)), dict(max_blocks=-1), dict(num_seqs=-1),
                dict(max_new=-1), dict(num_seqs=65536), dict(max_blocks=2**24)):
        refused(lib, lib.PKV_ERR_INVALID_ARG, _bounds(lib, **bad), "pkv_block_bounds")
    refused(lib, lib.PKV_ERR_UNSUPPORTED_SHAPE, _bounds(lib, kv=_kv(lib, 96)), "head_dim")
    for empty in (dict(num_seqs=0), dict(max_new=0), dict(max_blocks=0)):
        assert _bounds(lib, **empty) == lib.PKV_OK


def _select(lib, **kw):
    a = dict(bounds=FAKE, num_blocks=100, hkv=2, d=128, q=FAKE, hq=8, tables=FAKE, max_blocks=64,
             num_seqs=3, row_seq=FAKE, row_lens=FAKE, rows=5, max_len=1000, sink=1, recent=2,
             blocks=8, sel=FAKE, ws=FAKE, ws_bytes=1 << 20)
    a.update(kw)
    return lib._lib.pkv_select_blocks(*a.values(), None)


def test_select_blocks_refuses(lib):
    arg, shape = lib.PKV_ERR_INVALID_ARG, lib.PKV_ERR_UNSUPPORTED_SHAPE
    for bad in (dict(bounds=None), dict(q=None), dict(tables=None), dict(row_lens=None),
                dict(sel=None), dict(bounds=ctypes.c_void_p(0x3002)),
                dict(q=ctypes.c_void_p(0x3008)), dict(num_blocks=0), dict(hkv=0), dict(rows=-1),
                dict(num_seqs=-1), dict(max_blocks=-1), dict(blocks=-1), dict(max_len=-1),
                dict(blocks=0), dict(sink=-1), dict(recent=0), dict(sink=7), dict(recent=2**31 - 1),
                dict(row_seq=None), dict(max_len=1025), dict(rows=2**22 + 1),
                dict(max_len=2**20 + 1, max_blocks=2**17)):
        refused(lib, arg, _select(lib, **bad), "pkv_select_blocks")
    for bad in (dict(d=96), dict(hq=7), dict(hq=0), dict(hq=34)):
        refused(lib, shape, _select(lib, **bad), "pkv_select_blocks")
    need = lib.pkv_select_workspace_bytes(5, 8, 2, 128, 1000, 8)
    assert need >= 5 * 2 * 63 * 8
    for bad in (dict(ws=None), dict(ws_bytes=need - 1), dict(ws=ctypes.c_void_p(0x3004))):
        refused(lib, arg, _select(lib, **bad), "workspace")
    assert lib.pkv_select_workspace_bytes(5, 8, 2, 128, 128, 8) == 0  # every block is chosen
    assert lib.pkv_select_workspace_bytes(5, 8, 2, 128, 2**20 + 1, 8) == 0
    assert _select(lib, rows=0, q=None, sel=None) == lib.PKV_OK


def _sparse(lib, kv=None, **kw):
    a = dict(q=FAKE, hq=8, tables=FAKE, max_blocks=64, num_seqs=3, row_seq=FAKE, row_lens=FAKE,
             rows=5, sel=FAKE, blocks=8, scale=0.1, out=FAKE, lse=None, ws=FAKE, ws_bytes=1 << 30)
    a.update(kw)
    return lib._lib.pkv_sparse_attention(ctypes.byref(kv or _kv(lib)), *a.values(), None)


def test_sparse_attention_refuses(lib):
    arg, shape = lib.PKV_ERR_INVALID_ARG, lib.PKV_ERR_UNSUPPORTED_SHAPE
    for bad in (dict(q=None), dict(tables=None), dict(row_lens=None), dict(sel=None),
                dict(out=None), dict(q=ctypes.c_void_p(0x3008)), dict(out=ctypes.c_void_p(0x3004)),
                dict(rows=-1), dict(num_seqs=-1), dict(max_blocks=-1), dict(blocks=-1),
                dict(blocks=0), dict(blocks=65537), dict(scale=0.0), dict(scale=-1.0),
                dict(scale=float("nan")), dict(row_seq=None), dict(rows=2**22 + 1)):
        refused(lib, arg, _sparse(lib, **bad), "pkv_sparse_attention")
    for bad in (dict(hq=7), dict(hq=34), dict(kv=_kv(lib, 32)), dict(kv=_kv(lib, 128, 8))):
        refused(lib, shape, _sparse(lib, **bad), "pkv_sparse_attention")
    assert _sparse(lib, rows=0, q=None, sel=None, out=None) == lib.PKV_OK
    need = lib.pkv_sparse_workspace_bytes(1, 8, 2, 128, 4096)
    if need:
        for bad in (dict(ws=None), dict(ws_bytes=need - 1), dict(ws=ctypes.c_void_p(0x3004))):
            refused(lib, arg, _sparse(lib, rows=1, blocks=4096, **bad), "workspace")


def test_binding_refuses_host_tensors(lib):
    import torch
    if torch.cuda.is_available():
        pytest.skip("for a box without a GPU")
    with pytest.raises((TypeError, RuntimeError, AssertionError)):
        z = torch.zeros(1, dtype=torch.int32)
        lib.pkv_extend_tables(z.view(1, 1), z, z, z, z, z, torch.zeros(2, dtype=torch.int32), z, z,
                              0)


def test_tensor_address_takes_gpu_tensors_only():
    """The binding's look at a tensor (CPU side): anything but a tensor on the GPU asked for is None,
    wrong calls are TypeErrors."""
    import torch
    from paper_2607_23815_amd import _tensor_address as m
    t = torch.zeros((2, 3, 4), dtype=torch.bfloat16)
    for x in (t, t.transpose(0, 1), torch.zeros(0), t.to_sparse(), None, 3, "t",
              torch.empty((2, 3, 4), dtype=torch.bfloat16, device="meta")):
        assert m.address(x, torch.bfloat16, 0) is None
        assert m.rows_address(x, torch.bfloat16, 0, 2, 3, 4) is None
    assert m.address(t, "dtype", 0) is None
    for call, args in ((m.address, (t,)), (m.address, (t, t.dtype, None)),
                       (m.rows_address, (t, t.dtype, 0)), (m.rows_address, (t, t.dtype, 0, 2, "3", 4))):
        with pytest.raises(TypeError):
            call(*args)


def test_rope_spec_takes_no_number_of_axes_for_none(lib):
    assert lib.rope_spec([1.0] * 8, axis_of=[0, 2] * 4).num_axes == 3
    for n in (0, -1):
        refused(lib, lib.PKV_ERR_INVALID_ARG, _rope(lib, rope=lib.rope_spec([1.0] * 8, num_axes=n)),
                "num_axes")


def test_rope_append_refuses_frequencies_without_a_fraction(lib):
    """Angles past the fractions of 64 bits, or past their range (NaN), are refused."""
    for f in (1e300, -1e300, 2.0**20 * 1.001):
        refused(lib, lib.PKV_ERR_INVALID_ARG, _rope(lib, rope=lib.rope_spec([1.0] * 7 + [f])),
                "inv_freq")
    assert _rope(lib, rope=lib.rope_spec([-2.0**20, 2.0**20] * 4), rows=0) == lib.PKV_OK
