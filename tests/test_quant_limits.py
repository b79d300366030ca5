"""CPU tier: the sizes that the quantised cache's calls take, on both sides of their limits (no GPU is touched
here: a call that passes its checks ends at the launch)."""

import pytest

from tests.test_quant_abi import FAKE, _append, _blocks, _decode, _kv, _pool, lib, refused  # noqa: F401


def passes(lib, call, *args, **kw):  # noqa: F811
    """The call passes its checks, the launch's own among them, and finds no GPU."""
    import torch
    if torch.cuda.is_available():
        pytest.skip("the calls that pass would launch, on addresses that are none")
    assert call(lib, *args, **kw) == lib.PKV_ERR_HIP
    assert "invalid argument" not in lib.pkv_last_error(), lib.pkv_last_error()


@pytest.mark.parametrize("back", [0, 1])
@pytest.mark.parametrize("d", [64, 128])
def test_pairs_of_blocks(lib, back, d):  # noqa: F811
    """A wave takes a pair's kv head, four waves a workgroup, and a grid holds fewer than 2^32 threads: 2^26 - 4 items
    at most. What is refused is refused by the argument checks."""
    kv, pool = (lambda h: _kv(lib, head_dim=d, hkv=h)), (lambda h: _pool(lib, d, h))
    for heads, n in ((1, 2**26 - 3), (1, 2**26 - 1), (1, 2**26), (2, 2**25 - 1), (5, (2**26 - 4) // 5 + 1)):
        refused(lib, lib.PKV_ERR_INVALID_ARG, _blocks(lib, back, kv(heads), pool(heads), n=n), "2^26")
    for heads, n in ((1, 2**26 - 4), (2, 2**25 - 2), (5, (2**26 - 4) // 5)):
        passes(lib, _blocks, back, kv(heads), pool(heads), n=n)


def test_sequences_of_a_decode(lib):  # noqa: F811
    for heads, n in ((1, 2**22), (3, 2**22 // 3 + 1)):
        refused(lib, lib.PKV_ERR_INVALID_ARG, _decode(lib, _kv(lib, hkv=heads), hq=2 * heads, num_seqs=n), "2^22")
    for heads, n in ((1, 2**22 - 1), (3, (2**22 - 1) // 3)):
        for longest in (100, 1000, 9000, 2**30):
            passes(lib, _decode, _kv(lib, hkv=heads), hq=2 * heads, num_seqs=n, max_len=longest, max_blocks=2**26)


def test_blocks_of_an_append(lib):  # noqa: F811
    for heads in (1, 5):
        most = (((1 << 24) - 1) // heads - 2) * 16 + 15
        a = dict(ks=1024, vs=1024, max_blocks=2**30, num_seqs=65535)
        passes(lib, _append, _kv(lib, hkv=heads), max_new=most, **a)
        refused(lib, lib.PKV_ERR_INVALID_ARG, _append(lib, _kv(lib, hkv=heads), max_new=most + 1, **a), "2^24")


def test_a_decode_workspace_is_for_the_calls_own_sizes(lib):  # noqa: F811
    """Smaller calls can need more than larger ones. One that is given too little is refused, and the largest of
    several sizes' needs serves each of them."""
    size = lambda n, longest: lib.pkv_quant_decode_workspace_bytes(n, 32, 8, 128, 4, longest)
    call = lambda n, longest, ws, nbytes: _decode(lib, _kv(lib, hkv=8), hq=32, num_seqs=n, max_len=longest,
                                                  max_blocks=1024, ws=ws, ws_bytes=nbytes)
    assert size(128, 4096) == 0 < size(127, 4096)
    assert 0 < size(64, 9000) < size(64, 8192)
    for n, longest, given in ((127, 4096, 0), (64, 8192, size(64, 9000))):
        for ws in (None, FAKE):
            refused(lib, lib.PKV_ERR_INVALID_ARG, call(n, longest, ws, given), "workspace", "pkv_quant_decode_workspace_bytes")
    sizes = [(n, longest) for n in (1, 2, 7, 64, 127, 128, 300) for longest in (100, 2048, 2049, 8192, 9000, 16000)]
    most = max(size(*x) for x in sizes)
    for x in sizes:
        passes(lib, lambda lib: call(*x, FAKE, most))
