"""CPU tier: the calls of the quantised cache refuse bad arguments on the host, before any launch, and take
empty calls as successful no-ops (no GPU is touched here)."""
import ctypes

import pytest

from oracle import quant as Q


@pytest.fixture(scope="module")
def lib():
    from paper_2607_23815_amd import lib as L
    return L


FAKE = ctypes.c_void_p(0x3000)  # (host-side checks never dereference an address)


def refused(lib, status, got, *words):
    assert got == status, lib.pkv_last_error()
    for w in words:
        assert w in lib.pkv_last_error(), lib.pkv_last_error()


def _kv(lib, head_dim=128, bits=4, block_size=16, hkv=2, blocks=10, cache=0x1000):
    return lib.QuantKV(cache, blocks, block_size, hkv, head_dim, bits)


def _pool(lib, head_dim=128, hkv=2):
    return lib.PagedKV(0x1000, 0x2000, 10, 16, hkv, head_dim)


def _append(lib, kv=None, **kw):
    a = dict(k=FAKE, ks=256, v=FAKE, vs=256, tables=FAKE, max_blocks=4, cached=FAKE, cu=FAKE, num_seqs=2,
             total=5, max_new=3)
    a.update(kw)
    return lib._lib.pkv_quant_append(ctypes.byref(kv or _kv(lib)), *a.values(), None)


def _decode(lib, kv=None, **kw):
    a = dict(q=FAKE, hq=8, tables=FAKE, max_blocks=64, lens=FAKE, num_seqs=3, max_len=1000, scale=0.1,
             out=FAKE, lse=None, ws=FAKE, ws_bytes=1 << 30)
    a.update(kw)
    return lib._lib.pkv_quant_decode_attention(ctypes.byref(kv or _kv(lib)), *a.values(), None)


def _prefill(lib, kv=None, **kw):
    a = dict(q=FAKE, hq=8, tables=FAKE, max_blocks=1024, cached=FAKE, cu=FAKE, num_seqs=3, total=50,
             max_new=20, max_total=1000, scale=0.1, out=FAKE, lse=None, ws=None, ws_bytes=0)
    a.update(kw)
    return lib._lib.pkv_quant_prefill_attention(ctypes.byref(kv or _kv(lib)), *a.values(), None)


def _blocks(lib, back, kv=None, pool=None, pairs=FAKE, n=3):
    kv, pool = kv or _kv(lib), pool or _pool(lib)
    if back:
        return lib._lib.pkv_dequant_blocks(ctypes.byref(kv), ctypes.byref(pool), pairs, n, None)
    return lib._lib.pkv_quant_blocks(ctypes.byref(pool), ctypes.byref(kv), pairs, n, None)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bits", [4, 8])
def test_block_bytes(lib, d, bits):
    assert lib.pkv_quant_block_bytes(1, d, bits) == Q.slab_bytes(d, bits)
    assert lib.pkv_quant_block_bytes(7, d, bits) == 7 * Q.slab_bytes(d, bits)
    assert lib.pkv_quant_block_bytes(0, d, bits) == lib.pkv_quant_block_bytes(1, d, 5) == 0
    assert lib.pkv_quant_block_bytes(1, 96, bits) == 0
    t = lib.alloc_quant_cache(3, 2, d, bits, device="cpu")
    assert t.shape == (3, 2, Q.slab_bytes(d, bits))
    with pytest.raises(ValueError):
        lib.alloc_quant_cache(3, 2, d, 6, device="cpu")


@pytest.mark.parametrize("call", [_append, _decode, _prefill, lambda lib, kv: _blocks(lib, 0, kv),
                                  lambda lib, kv: _blocks(lib, 1, kv)])
def test_caches_refused(lib, call):
    shape, arg = lib.PKV_ERR_UNSUPPORTED_SHAPE, lib.PKV_ERR_INVALID_ARG
    refused(lib, shape, call(lib, _kv(lib, head_dim=96)), "head_dim")
    refused(lib, shape, call(lib, _kv(lib, bits=5)), "bits")
    refused(lib, shape, call(lib, _kv(lib, bits=16)), "bits")
    refused(lib, shape, call(lib, _kv(lib, block_size=32)), "block_size")
    refused(lib, arg, call(lib, _kv(lib, cache=None)), "cache is NULL")
    refused(lib, arg, call(lib, _kv(lib, cache=0x1008)), "aligned")
    refused(lib, arg, call(lib, _kv(lib, blocks=0)), "num_blocks")
    refused(lib, arg, call(lib, _kv(lib, hkv=0)), "num_kv_heads")


def test_null_caches(lib):
    arg, none = lib.PKV_ERR_INVALID_ARG, [None] * 20
    L = lib._lib
    pool = ctypes.byref(_pool(lib))
    refused(lib, arg, L.pkv_quant_append(None, FAKE, 0, FAKE, 0, *none[:1], 0, None, None, 0, 0, 0, None), "NULL")
    refused(lib, arg, L.pkv_quant_blocks(pool, None, FAKE, 1, None), "NULL")
    refused(lib, arg, L.pkv_dequant_blocks(None, pool, FAKE, 1, None), "NULL")
    refused(lib, arg, L.pkv_quant_blocks(None, ctypes.byref(_kv(lib)), FAKE, 1, None), "NULL")


@pytest.mark.parametrize("bad", [
    dict(k=None), dict(v=None), dict(tables=None), dict(cached=None), dict(cu=None),
    dict(k=ctypes.c_void_p(0x3008)), dict(v=ctypes.c_void_p(0x3002)), dict(ks=248), dict(vs=260),
    dict(ks=-256), dict(num_seqs=-1), dict(total=-1), dict(max_new=-1), dict(max_new=0), dict(max_blocks=0),
    dict(max_blocks=-1), dict(num_seqs=65536), dict(max_new=2**30)])
def test_append_refuses(lib, bad):
    refused(lib, lib.PKV_ERR_INVALID_ARG, _append(lib, **bad), "pkv_quant_append")


def test_blocks_refuse(lib):
    arg = lib.PKV_ERR_INVALID_ARG
    for back in (0, 1):
        refused(lib, arg, _blocks(lib, back, pairs=None), "NULL")
        refused(lib, arg, _blocks(lib, back, n=-1), "negative")
        refused(lib, arg, _blocks(lib, back, n=2**26), "2^26")
        refused(lib, arg, _blocks(lib, back, pool=_pool(lib, 64)), "differ")
        refused(lib, arg, _blocks(lib, back, pool=_pool(lib, 128, 4)), "differ")
        refused(lib, lib.PKV_ERR_UNSUPPORTED_SHAPE, _blocks(lib, back, pool=_pool(lib, 32)), "head_dim")
        assert _blocks(lib, back, pairs=None, n=0) == lib.PKV_OK


def test_decode_refuses(lib):
    arg, shape = lib.PKV_ERR_INVALID_ARG, lib.PKV_ERR_UNSUPPORTED_SHAPE
    for bad in (dict(q=None), dict(tables=None), dict(lens=None), dict(out=None),
                dict(q=ctypes.c_void_p(0x3008)), dict(out=ctypes.c_void_p(0x3004)), dict(num_seqs=-1),
                dict(max_len=-1), dict(max_len=0), dict(max_blocks=-1), dict(max_blocks=0),
                dict(max_len=1025), dict(scale=0.0), dict(scale=float("nan")), dict(scale=-1.0),
                dict(num_seqs=2**21 + 1)):
        refused(lib, arg, _decode(lib, **bad), "pkv_quant_decode_attention")
    refused(lib, arg, _decode(lib, num_seqs=1, max_len=2**30 + 1, max_blocks=2**27), "2^30")
    for bad in (dict(hq=7), dict(hq=0), dict(hq=34)):
        refused(lib, shape, _decode(lib, **bad), "num_q_heads")
    need = lib.pkv_quant_decode_workspace_bytes(1, 8, 2, 128, 4, 2**20)
    assert need > 0
    for bad in (dict(ws=None), dict(ws_bytes=need - 1), dict(ws=ctypes.c_void_p(0x3004))):
        refused(lib, arg, _decode(lib, num_seqs=1, max_len=2**20, max_blocks=2**16, **bad), "workspace")
    assert _decode(lib, num_seqs=0, q=None, out=None, lens=None) == lib.PKV_OK
    for n in ((0, 8, 2, 128, 4, 10), (1, 8, 3, 128, 4, 10), (1, 8, 2, 128, 4, 0), (2**21 + 1, 8, 2, 128, 4, 10)):
        assert lib.pkv_quant_decode_workspace_bytes(*n) == 0


def test_prefill_refuses(lib):
    arg, shape = lib.PKV_ERR_INVALID_ARG, lib.PKV_ERR_UNSUPPORTED_SHAPE
    for bad in (dict(q=None), dict(tables=None), dict(cached=None), dict(cu=None), dict(out=None),
                dict(q=ctypes.c_void_p(0x3008)), dict(num_seqs=-1), dict(total=-1), dict(max_new=0),
                dict(max_total=19), dict(max_blocks=62), dict(scale=0.0), dict(num_seqs=65536)):
        refused(lib, arg, _prefill(lib, **bad), "pkv_quant_prefill_attention")
    refused(lib, shape, _prefill(lib, hq=7), "num_q_heads")
    refused(lib, arg, _prefill(lib, max_total=2**30 + 1, max_blocks=2**27), "2^30")
    long = dict(num_seqs=1, max_total=16000)
    need = lib.pkv_quant_prefill_workspace_bytes(1, 50, 8, 2, 128, 4, 20, 16000)
    assert need > 0
    for bad in (dict(ws=FAKE, ws_bytes=need - 1), dict(ws=ctypes.c_void_p(0x3004), ws_bytes=need)):
        refused(lib, arg, _prefill(lib, **long, **bad), "workspace")
    assert _prefill(lib, total=0, q=None, out=None) == lib.PKV_OK
    assert lib.pkv_quant_prefill_workspace_bytes(1, 50, 8, 2, 128, 5, 20, 16000) == 0


def test_binding_refuses_host_tensors(lib):
    import torch
    if torch.cuda.is_available():
        pytest.skip("for a box without a GPU")
    t = lib.alloc_quant_cache(3, 2, 64, 4, device="cpu")
    with pytest.raises((TypeError, RuntimeError, AssertionError)):
        lib.pkv_dequant_blocks(t, t, t, torch.zeros((1, 2), dtype=torch.int32))
