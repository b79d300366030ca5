"""CPU tier: the sizes that the quantised cache's calls take, on both sides of their limits (no GPU is touched
here: a call that passes its checks ends at the launch)."""

import pytest

from tests.test_quant_abi import _append, _blocks, _decode, _kv, _pool, lib, refused  # noqa: F401


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
