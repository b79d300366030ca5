"""GPU tier: attention over the quantised cache where a tile, a wave or an address could go wrong unseen: every new row
of a prefill (all column tiles and waves of a workgroup), decodes whose items are one wave each, merges of more than
64 splits, a pool behind 2^32 bytes, and queries whose dims lie far apart beside 4-bit keys. Definitions in 64 bits;
tolerances are those that test_gpu_quant_attention derives."""
import numpy as np
import pytest

from oracle import quant as Q
from tests.gpu_util import bf16_to_f64, i32, say, to_dev_bits, to_host_bits
from tests.paged_fixture import rand_bf16
from tests.test_gpu_quant_attention import check_decode, parts_off, pool, rows_of, sequence

pytestmark = pytest.mark.gpu


def check_all_rows(lib, rng, cached, new, hq, hkv, d, bits, q=None, plan=True):
    import torch
    cached, new = np.array(cached), np.array(new)
    lens, cu = cached + new, np.concatenate([[0], np.cumsum(new)])
    tables, host = pool(rng, lens.tolist(), hkv, d, bits)
    t, b, g = int(new.sum()), len(new), hq // hkv
    q = rand_bf16(rng, (t, hq, d)) if q is None else q
    out = torch.full((t, hq, d), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((t, hq), 7.0, device="cuda")
    sizes = int(new.max()), int(lens.max())
    need = lib.pkv_quant_prefill_workspace_bytes(b, t, hq, hkv, d, bits, *sizes)
    scale = d ** -0.5
    lib.pkv_quant_prefill_attention(torch.from_numpy(host).cuda(), to_dev_bits(q), i32(tables), i32(cached), i32(cu), *sizes,
                                    scale, out, lse=lse, workspace=lib.alloc_workspace(need) if plan else None)
    got, got_lse = bf16_to_f64(to_host_bits(out)), lse.double().cpu().numpy()
    worst = 0.0
    for i in range(b):
        if new[i] == 0:
            continue
        k, v = sequence(host, tables[i], int(lens[i]), d, bits)
        for j in range(new[i]):
            n, row = int(cached[i]) + j + 1, cu[i] + j
            for h in range(hkv):
                rows = slice(h * g, h * g + g)
                x = bf16_to_f64(q[row, rows])
                o, z, tol, tol_z = rows_of(x, k[h, :n], v[h, :n], scale, 2.0**-8, parts_off(x, bits))
                err = np.abs(got[row, rows] - o)
                assert (err <= tol).all(), (i, j, h, float((err / tol).max()))
                assert (np.abs(got_lse[row, rows] - z) <= tol_z).all(), (i, j, h)
                worst = max(worst, float((err / np.maximum(tol, 1e-300)).max()))
    say(f"  prefill {hq}/{hkv} heads of {d}, bits {bits}, {t} rows: {worst:.2f} of the tolerance")
    return need


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("hq,hkv,d", [(4, 2, 64), (8, 2, 128), (3, 3, 128), (20, 1, 64), (32, 8, 128)])
def test_prefill_every_row(gpu_lib, hq, hkv, d, bits):
    rng = np.random.default_rng(1000 + hq + d + bits)
    say(f"[quant rows] {hq}/{hkv} heads of {d}, bits {bits}")
    check_all_rows(gpu_lib, rng, [0, 5, 16, 63, 64, 130, 0], [1, 3, 0, 70, 64, 37, 150], hq, hkv, d, bits)
    check_all_rows(gpu_lib, rng, [70, 200, 1], [130, 1, 65], hq, hkv, d, bits, plan=False)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("d", [64, 128])
def test_prefill_every_row_of_splits(gpu_lib, bits, d):
    """Splits of 768 keys, which begin and end among the rows' last keys."""
    rng = np.random.default_rng(2000 + d + bits)
    say(f"[quant rows] splits, heads of {d}, bits {bits}")
    hq, hkv, new = 4, 2, [60, 33, 90]
    need = check_all_rows(gpu_lib, rng, [740, 2290, 1500], new, hq, hkv, d, bits)
    assert need // (sum(new) * hq * (d + 2) * 4) == 4  # (2323 keys)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("d", [64, 128])
def test_prefill_long_batches_are_split(gpu_lib, bits, d):
    """The batches of test_prefill_long: splits of 768 keys, 6 and 11."""
    for seqs, new, hq, hkv, longest, splits in ((3, [33, 70, 1], 4, 2, 4033, 6),
                                                (23, [9, 70, 1] + [5] * 20, 4, 1, 8309, 11)):
        need = gpu_lib.pkv_quant_prefill_workspace_bytes(seqs, sum(new), hq, hkv, d, bits, max(new), longest)
        assert need // (sum(new) * hq * (d + 2) * 4) == splits


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("g", [4, 8, 16])
def test_decode_one_wave_an_item(gpu_lib, bits, d, g):
    """2048 (sequence, kv head) pairs and more, of short lengths."""
    rng = np.random.default_rng(bits + d + g)
    lens = [int(n) for n in rng.integers(0, 50, 257)]
    lens[7], lens[100] = 300, 512
    check_decode(gpu_lib, rng, lens, 8 * g, 8, d, bits)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("n,hq,d", [(40000, 2, 64), (131072, 4, 128), (70001, 16, 64)])
def test_decode_of_many_splits(gpu_lib, bits, n, hq, d):
    """One kv head, 79 to 128 splits: the merge's second round of 64."""
    lib = gpu_lib
    need = lib.pkv_quant_decode_workspace_bytes(1, hq, 1, d, bits, n)
    assert 64 < need // (hq * (d + 2) * 4) <= 128
    check_decode(lib, np.random.default_rng(n + bits), [n], hq, 1, d, bits)


@pytest.mark.parametrize("bits", [4, 8])
def test_a_pool_behind_32_bits(gpu_lib, bits):
    """Blocks whose bytes lie past 2^32: the same bits as from the same blocks in a small pool."""
    import torch
    lib = gpu_lib
    rng = np.random.default_rng(bits)
    hq, hkv, d, cached, new = 16, 4, 128, 700, 30
    n = cached + new
    tables, host = pool(rng, [n], hkv, d, bits)
    small = torch.from_numpy(host).cuda()
    used = small.shape[0]
    blocks = (1 << 32) // (hkv * Q.slab_bytes(d, bits)) + 2 * used
    say(f"[quant rows] {blocks} blocks, bits {bits}")
    large = lib.alloc_quant_cache(blocks, hkv, d, bits)
    first = blocks - used
    assert first * hkv * Q.slab_bytes(d, bits) > 1 << 32
    large[first:] = small
    large[:used] = 255  # (where addresses cut to 32 bits would point to)
    cut = (first * hkv * Q.slab_bytes(d, bits) & 0xFFFFFFFF) // (hkv * Q.slab_bytes(d, bits))
    large[cut:cut + 2 * used] = 255
    q = to_dev_bits(rand_bf16(rng, (new, hq, d)))
    for call in ("decode", "prefill"):
        outs = []
        for cache, table in ((small, tables), (large, np.where(tables < 0, tables, tables + first))):
            rows = 1 if call == "decode" else new
            out = torch.empty((rows, hq, d), dtype=torch.bfloat16, device="cuda")
            if call == "decode":
                lib.pkv_quant_decode_attention(cache, q[:1], i32(table), i32([n]), n, 0.1, out)
            else:
                lib.pkv_quant_prefill_attention(cache, q, i32(table), i32([cached]), i32([0, new]), new, n, 0.1, out)
            outs.append(out)
        assert torch.isfinite(outs[0]).all() and torch.equal(outs[0].view(torch.int16), outs[1].view(torch.int16))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("most", [2.0**5, 2.0**9])
def test_prefill_queries_far_apart(gpu_lib, d, most):
    """In each group of 32 dims one query is much larger than the others, whose parts end at 2^-14 of it. (The scores
    stay below what a row of ordinary queries has: the large dim is on the scale of one, the others below.)"""
    rng = np.random.default_rng(d + int(most))
    rows, hq, hkv = 90, 8, 2
    x = bf16_to_f64(rand_bf16(rng, (rows, hq, d)))
    at = rng.integers(0, 32, (rows, hq, d // 32))
    small = x / most
    for group in range(d // 32):
        r, h = np.ogrid[:rows, :hq]
        small[r, h, 32 * group + at[..., group]] = np.sign(x[r, h, 32 * group + at[..., group]]) * 4.0
    q = (small.astype(np.float32).view(np.uint32) >> 16).astype(np.uint16)
    off = parts_off(bf16_to_f64(q), 4)
    assert (off > 0).mean() > (0.9 if most > 100 else 0.2)
    check_all_rows(gpu_lib, rng, [100, 300], [50, 40], hq, hkv, d, 4, q=q)
