"""GPU tier: calls of the quantised cache that its documentation allows at the edges: nothing to do, one row however its
strides read, bounds far above every length, blocks that several sequences share, the same pool block in several pairs,
large groups of query heads."""
import numpy as np
import pytest

from oracle import quant as Q
from tests.gpu_util import bf16_to_f64, i32, to_dev_bits
from tests.paged_fixture import rand_bf16
from tests.test_gpu_quant_attention import BS, check_prefill, pool

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [4, 8])
def test_nothing_to_do(gpu_lib, bits):
    import torch
    lib = gpu_lib
    hq, hkv, d = 4, 2, 64
    cache = lib.alloc_quant_cache(3, hkv, d, bits).fill_(9)
    k, v = (torch.full(s, 3.0, dtype=torch.bfloat16, device="cuda") for s in ((3, hkv, d // 8, BS, 8), (3, hkv, d, BS)))
    rows = lambda n, h: torch.zeros((n, h, d), dtype=torch.bfloat16, device="cuda")
    table = i32(np.zeros((2, 4)))
    lib.pkv_quant_append(cache, rows(0, hkv), rows(0, hkv), table, i32([0, 5]), i32([0, 0, 0]), 0)
    lib.pkv_quant_append(cache, rows(0, hkv), rows(0, hkv), table[:0], i32([]), i32([0]), 0)
    lib.pkv_quant_append(cache, rows(2, hkv), rows(2, hkv), table, i32([0, 5]), i32([0, 0, 0]), 2)  # (rows of nobody)
    lib.pkv_quant_blocks(k, v, cache, i32(np.zeros((0, 2))))
    lib.pkv_dequant_blocks(cache, k, v, i32(np.zeros((0, 2))))
    lib.pkv_quant_decode_attention(cache, rows(0, hq), table[:0], i32([]), 10, 1.0, rows(0, hq))
    lib.pkv_quant_prefill_attention(cache, rows(0, hq), table, i32([0, 5]), i32([0, 0, 0]), 0, 5, 1.0, rows(0, hq))
    out = torch.full((2, hq, d), 7.0, dtype=torch.bfloat16, device="cuda")
    lib.pkv_quant_prefill_attention(cache, rows(2, hq), table, i32([0, 5]), i32([0, 0, 0]), 2, 60, 1.0, out)
    torch.cuda.synchronize()
    assert (cache == 9).all() and (k == 3).all() and (v == 3).all() and (out == 7).all()


@pytest.mark.parametrize("bits", [4, 8])
def test_one_row_whose_strides_say_little(gpu_lib, bits):
    """[1][heads][dim] as a transposed view: its rows' stride is dim and means nothing."""
    import torch
    lib = gpu_lib
    rng = np.random.default_rng(bits)
    hkv, d = 3, 64
    k, v = (to_dev_bits(rand_bf16(rng, (hkv, 1, d))).transpose(0, 1) for _ in range(2))
    assert k.stride(0) == d
    a, b = (lib.alloc_quant_cache(2, hkv, d, bits).fill_(255) for _ in range(2))
    args = i32([[1]]), i32([6]), i32([0, 1]), 1
    lib.pkv_quant_append(a, k, v, *args)
    lib.pkv_quant_append(b, k.clone(memory_format=torch.contiguous_format), v.contiguous(), *args)
    assert torch.equal(a, b) and not (a[1] == 255).all()
    with pytest.raises(ValueError):  # two rows are not such a view
        lib.pkv_quant_append(a, to_dev_bits(rand_bf16(rng, (hkv, 2, d))).transpose(0, 1), v.expand(2, hkv, d), *args[:2],
                             i32([0, 2]), 2)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("d", [64, 128])
def test_prefill_bounds_far_above_the_lengths(gpu_lib, bits, d):
    """As in a captured step: bounds for 20000 keys, splits and their merge included, over lengths from one to a split's;
    the bits of the call with tight bounds."""
    import torch
    lib = gpu_lib
    rng = np.random.default_rng(bits + d)
    hq, hkv = 8, 2
    cached, new = np.array([0, 700, 40, 0, 300]), np.array([1, 20, 0, 33, 5])
    tables, host = pool(rng, (cached + new).tolist(), hkv, d, bits)
    wide = np.full((5, 1250), -1, np.int32)
    wide[:, :tables.shape[1]] = tables
    cache, t = torch.from_numpy(host).cuda(), int(new.sum())
    q = to_dev_bits(rand_bf16(rng, (t, hq, d)))
    cu = i32(np.concatenate([[0], np.cumsum(new)]))
    outs = []
    for table, most, longest in ((tables, 33, 720), (wide, 33, 20000), (wide, 400, 20000)):
        need = lib.pkv_quant_prefill_workspace_bytes(5, t, hq, hkv, d, bits, most, longest)
        assert longest < 20000 or need > 2 * t * hq * (d + 2) * 4
        ws = torch.full((max(need, 16),), 255, dtype=torch.uint8, device="cuda")
        out, lse = torch.empty((t, hq, d), dtype=torch.bfloat16, device="cuda"), torch.empty((t, hq), device="cuda")
        lib.pkv_quant_prefill_attention(cache, q, i32(table), i32(cached), cu, most, longest, 0.1, out, lse=lse, workspace=ws)
        outs.append((out, lse))
    for out, lse in outs[1:]:
        assert torch.equal(out.view(torch.int16), outs[0][0].view(torch.int16)) and torch.equal(lse, outs[0][1])


@pytest.mark.parametrize("bits", [4, 8])
def test_sequences_share_their_prefix_blocks(gpu_lib, bits):
    """Four sequences over one parked prefix, each with a last block of its own: appends leave the shared blocks, and
    equal suffixes give equal rows."""
    import torch
    lib = gpu_lib
    rng = np.random.default_rng(bits)
    hq, hkv, d, prefix = 8, 2, 128, 40
    cache = lib.alloc_quant_cache(prefix + 5, hkv, d, bits).fill_(255)
    k = to_dev_bits(rand_bf16(rng, (prefix, hkv, d // 8, BS, 8)))
    v = to_dev_bits(rand_bf16(rng, (prefix, hkv, d, BS)))
    at = rng.permutation(prefix + 5).astype(np.int32)
    lib.pkv_quant_blocks(k, v, cache, i32(np.stack([np.arange(prefix), at[:prefix]], 1)))
    before = cache.clone()
    tables = np.stack([np.append(at[:prefix], at[prefix + i]) for i in range(4)])
    cached, cu = i32([prefix * BS] * 4), i32([0, 3, 6, 9, 12])
    row = lambda h: to_dev_bits(np.tile(rand_bf16(rng, (3, h, d)), (4, 1, 1)))
    kn, vn, q = row(hkv), row(hkv), row(hq)
    lib.pkv_quant_append(cache, kn, vn, i32(tables), cached, cu, 3)
    shared = torch.from_numpy(at[:prefix].astype(np.int64)).cuda()
    assert torch.equal(cache[shared], before[shared])
    out = torch.empty((12, hq, d), dtype=torch.bfloat16, device="cuda")
    n = prefix * BS + 3
    lib.pkv_quant_prefill_attention(cache, q, i32(tables), cached, cu, 3, n, 0.1, out)
    last = torch.empty((4, hq, d), dtype=torch.bfloat16, device="cuda")
    lib.pkv_quant_decode_attention(cache, q[2::3].contiguous(), i32(tables), i32([n] * 4), n, 0.1, last)
    assert torch.isfinite(out).all() and torch.isfinite(last).all()
    for i in range(1, 4):
        assert torch.equal(out[3 * i:3 * i + 3].view(torch.int16), out[:3].view(torch.int16))
        assert torch.equal(last[i].view(torch.int16), last[0].view(torch.int16))


@pytest.mark.parametrize("bits", [4, 8])
def test_one_block_to_several(gpu_lib, bits):
    """A block may be named as a source more than once."""
    import torch
    lib = gpu_lib
    rng = np.random.default_rng(bits)
    hkv, d = 2, 64
    x = bf16_to_f64(rand_bf16(rng, (2, 1, hkv, BS, d)))
    cache = torch.from_numpy(np.concatenate([Q.blocks(x[0], x[1], d, bits)] * 2)).cuda()
    k, v = (torch.zeros(s, dtype=torch.bfloat16, device="cuda") for s in ((4, hkv, d // 8, BS, 8), (4, hkv, d, BS)))
    lib.pkv_dequant_blocks(cache, k, v, i32([[0, 3], [0, 1], [1, 0]]))
    for t in (k, v):
        assert torch.equal(t[3], t[1]) and torch.equal(t[3], t[0]) and (t[2] == 0).all() and (t[3] != 0).any()
    to = lib.alloc_quant_cache(3, hkv, d, bits).fill_(7)
    lib.pkv_quant_blocks(k, v, to, i32([[3, 2], [3, 0]]))
    assert torch.equal(to[0], to[2]) and (to[1] == 7).all()


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("hq,hkv,d", [(32, 1, 64), (48, 1, 128), (256, 2, 64)])
def test_prefill_large_groups(gpu_lib, bits, hq, hkv, d):
    """More query heads to a kv head than a wave has columns, or a workgroup; a group's columns in several tiles."""
    rng = np.random.default_rng(hq + bits)
    check_prefill(gpu_lib, rng, [50, 0, 200], [3, 20, 9], hq, hkv, d, bits)
