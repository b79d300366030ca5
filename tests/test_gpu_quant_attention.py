"""GPU tier: attention over the quantised cache.

Decode against its definition in 64 bits on what the codes stand for. Tolerance, per output element, from
the roundings on the way: a score is a 32-bit sum of D products, off by delta = (D + 8) 2^-24 scale
sum_d |q_d k_d| at most, a weight by 2 delta relative after the normalisation and by 2^-16 in two bf16 parts;
the output is rounded to bf16, half a step 2^-8:
    |error| <= (2^-16 + 2 delta + (n + 16) 2^-23) sum_p w_p |v_p| + 2^-8 |out|,
(n + 16) 2^-23 for the sums over n keys, the exponential, the value scale's product and the merges in 32 bits.
The LSE: delta + n 2^-24 and 2^-20 (1 + |lse|) for exp2, log2 and the result's own roundings.

Prefill against the same definition; there a weight times its token's value scale is rounded to bf16 once, which
is 2^-8 in the place of 2^-16, and queries beside 4-bit keys are taken in parts (parts_off)."""
import math

import numpy as np
import pytest

from oracle import quant as Q
from tests.gpu_util import bf16_to_f64, i32, say, to_dev_bits, to_host_bits
from tests.paged_fixture import rand_bf16

pytestmark = pytest.mark.gpu

BS = 16


def pool(rng, lens, hkv, d, bits):
    """Tables in random order, and a cache whose other blocks and tail slots are bytes of 255 (NaN)."""
    counts = [-(-n // BS) for n in lens]
    nb = sum(counts) + 3
    perm = rng.permutation(nb)
    tables = np.full((len(lens), max(counts) + 1), -1, np.int32)
    cache = np.full((nb, hkv, Q.slab_bytes(d, bits)), 255, np.uint8)
    at = 0
    for i, (n, c) in enumerate(zip(lens, counts)):
        mine = perm[at:at + c]
        at += c
        tables[i, :c] = mine
        if c == 0:
            continue
        x = bf16_to_f64(rand_bf16(rng, (2, c, hkv, BS, d)))
        cache[mine] = Q.blocks(x[0] * 2, x[1] * 2.0 ** rng.integers(-6, 6, (c, hkv, BS, 1)), d, bits)
        if n % BS:
            k, e, v, s = (y.copy() for y in Q.parts(cache[mine[-1]], d, bits))
            full = 15 if bits == 4 else 255
            k[:, n % BS:], e[:, n % BS:], v[:, n % BS:], s[:, n % BS:] = full, 255, full, np.nan
            cache[mine[-1]] = Q.joined(k, e, v, s, d, bits)
    return tables, cache


def sequence(cache, table, n, d, bits):
    """[hkv][n][d] keys and values."""
    k, v = Q.stands_for(cache[table[:-(-n // BS)]], d, bits)
    hkv = cache.shape[1]
    return (x.transpose(1, 0, 2, 3).reshape(hkv, -1, d)[:, :n] for x in (k, v))


def rows_of(q, k, v, scale, weight_off, query_off=0.0):
    """q [g][d], taken query_off [g][d] off at most, over k, v [n][d]: outputs, LSEs, and the elements' tolerances."""
    n, d = k.shape
    z = scale * q @ k.T
    delta = scale * (((d + 8) * 2.0**-24 * np.abs(q) + query_off) @ np.abs(k).T).max(1, keepdims=True)
    top = z.max(1, keepdims=True)
    w = np.exp(z - top)
    total = w.sum(1, keepdims=True)
    w /= total
    out, lse = w @ v, (top + np.log(total))[:, 0]
    tol = (weight_off + 2 * delta + (n + 16) * 2.0**-23) * (w @ np.abs(v)) + 2.0**-8 * np.abs(out)
    return out, lse, tol, delta[:, 0] + n * 2.0**-24 + 2.0**-20 * (1 + np.abs(lse))


def check_decode(lib, rng, lens, hq, hkv, d, bits, max_len=None, cut=None, nan_at=None):
    import torch
    tables, cache = pool(rng, lens, hkv, d, bits)
    b = len(lens)
    max_len = max_len or max(max(lens), 1)
    width = max(tables.shape[1], -(-max_len // BS))
    tables = np.pad(tables, ((0, 0), (0, width - tables.shape[1])), constant_values=-1)
    q = rand_bf16(rng, (b, hq, d))
    scale = 1 / math.sqrt(d)
    out = torch.full((b + 1, hq, d), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((b + 1, hq), 7.0, device="cuda")
    need = lib.pkv_quant_decode_workspace_bytes(b, hq, hkv, d, bits, max_len)
    ws = torch.full((need + 64,), 255, dtype=torch.uint8, device="cuda") if need else None
    args = torch.from_numpy(cache).cuda(), to_dev_bits(q), i32(tables), i32(lens), max_len, scale
    lib.pkv_quant_decode_attention(*args, out[:b], lse=lse[:b], workspace=None if ws is None else ws[:need])
    torch.cuda.synchronize()
    assert (out[b] == 7).all() and (lse[b] == 7).all() and (ws is None or (ws[need:] == 255).all())
    got, got_lse = bf16_to_f64(to_host_bits(out[:b])), lse[:b].double().cpu().numpy()
    again = torch.empty_like(out)
    lib.pkv_quant_decode_attention(*args, again[:b])  # (without an LSE, with a workspace of its own)
    assert torch.equal(again[:b].view(torch.int16), out[:b].view(torch.int16))
    worst = 0.0
    g = hq // hkv
    for i, n in enumerate(lens):
        n = min(n, max_len)
        if n <= 0:
            assert (got[i] == 0).all() and (got_lse[i] == -np.inf).all()
            continue
        k, v = sequence(cache, tables[i], n, d, bits)
        for h in range(hkv):
            rows = slice(h * g, h * g + g)
            o, z, tol, tol_z = rows_of(bf16_to_f64(q[i, rows]), k[h], v[h], scale, 2.0**-16)
            err = np.abs(got[i, rows] - o)
            assert (err <= tol).all(), (i, n, h, float((err / tol).max()))
            assert (np.abs(got_lse[i, rows] - z) <= tol_z).all(), (i, n, h)
            worst = max(worst, float((err / np.maximum(tol, 1e-300)).max()))
    say(f"  decode {hq}/{hkv} heads of {d}, bits {bits}, lens {lens[:6]}: {worst:.2f} of the tolerance")


HEADS = [(4, 4, 128), (8, 2, 64), (16, 2, 128), (7, 1, 64), (28, 4, 128), (16, 1, 64), (9, 1, 128), (32, 8, 128)]


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("hq,hkv,d", HEADS)
def test_decode(gpu_lib, hq, hkv, d, bits):
    rng = np.random.default_rng(hq + d + bits)
    check_decode(gpu_lib, rng, [1, 2, 15, 16, 17, 0, 63, 64, 65, 100, 255, 256, 257, 700], hq, hkv, d, bits)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (16, 4, 64), (16, 1, 128)])
def test_decode_long(gpu_lib, hq, hkv, d, bits):
    """Splits, whose last is short or missing, and table chunks of 1024 keys."""
    rng = np.random.default_rng(hq + d + bits + 1)
    check_decode(gpu_lib, rng, [5003], hq, hkv, d, bits)
    check_decode(gpu_lib, rng, [1, 9001, 1024, 4097, 0, 2048], hq, hkv, d, bits)
    check_decode(gpu_lib, rng, [30, 70], hq, hkv, d, bits, max_len=20000)  # a bound far above


def test_decode_lengths_past_the_bound(gpu_lib):
    rng = np.random.default_rng(3)
    check_decode(gpu_lib, rng, [500, 129, 128, 3], 8, 2, 64, 4, max_len=128)
    check_decode(gpu_lib, rng, [5000, 4000], 4, 2, 128, 8, max_len=4100)


def test_decode_many_sequences(gpu_lib):
    rng = np.random.default_rng(4)
    check_decode(gpu_lib, rng, [int(n) for n in rng.integers(0, 60, 700)], 8, 4, 64, 4)
    check_decode(gpu_lib, rng, [int(n) for n in rng.integers(1, 900, 130)], 4, 2, 64, 8)


@pytest.mark.parametrize("seqs", [70, 600])
def test_decode_splits_of_many_sequences(gpu_lib, seqs):
    """Items found in rounds of 64 sequences, and past the number that is looked through."""
    rng = np.random.default_rng(seqs)
    lens = [int(n) for n in rng.integers(0, 40, seqs)]
    for i in rng.choice(seqs, 4, replace=False):
        lens[i] = int(rng.integers(3000, 9500))
    check_decode(gpu_lib, rng, lens, 2, 1, 64, 4, max_len=9500)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("n", [40, 3000])
def test_decode_nan_keys_and_values(gpu_lib, bits, n):
    """A group that reads back as NaN makes NaN of the heads of its kv head, and of no other; behind the
    sequence's end, and in slots past it, it makes none."""
    import torch
    lib = gpu_lib
    rng = np.random.default_rng(bits + n)
    hq, hkv, d = 8, 4, 128
    tables, clean = pool(rng, [n, n, n], hkv, d, bits)
    q = to_dev_bits(rand_bf16(rng, (3, hq, d)))
    args = i32(tables), i32([n, n, n]), n, 0.1
    out = torch.empty((3, hq, d), dtype=torch.bfloat16, device="cuda")
    lib.pkv_quant_decode_attention(torch.from_numpy(clean).cuda(), q, *args, out)
    assert torch.isfinite(out).all()
    for part in (1, 3):  # key scales, value scales
        cache = clean.copy()
        block, slot = tables[1, (n - 3) // BS], (n - 3) % BS
        parts = [x.copy() for x in Q.parts(cache[block], d, bits)]
        parts[part][2, slot] = 255 if part == 1 else np.nan
        cache[block] = Q.joined(*parts, d, bits)
        hurt = torch.empty_like(out)
        lib.pkv_quant_decode_attention(torch.from_numpy(cache).cuda(), q, *args, hurt)
        assert torch.isnan(hurt[1, 4:6]).all()
        hurt[1, 4:6] = out[1, 4:6]
        assert torch.equal(hurt.view(torch.int16), out.view(torch.int16))


def test_decode_queries_that_are_not_finite(gpu_lib):
    import torch
    lib = gpu_lib
    rng = np.random.default_rng(8)
    hq, hkv, d, bits, n = 8, 2, 64, 4, 200
    tables, cache = pool(rng, [n, n], hkv, d, bits)
    q = rand_bf16(rng, (2, hq, d))
    q[0, 1, 5], q[1, 6, 7] = 0x7F80, 0x7FC0
    out = torch.empty((2, hq, d), dtype=torch.bfloat16, device="cuda")
    lib.pkv_quant_decode_attention(torch.from_numpy(cache).cuda(), to_dev_bits(q), i32(tables), i32([n, n]), n, 0.1,
                                   out)
    bad = torch.isnan(out).any(2).cpu().numpy()
    assert bad[0, 1] and bad[1, 6] and bad.sum() == 2


@pytest.mark.parametrize("bits", [4, 8])
def test_decode_extreme_scales(gpu_lib, bits):
    """Values near the largest and the least, and scores far apart: no sum leaves the 32-bit range."""
    import torch
    lib = gpu_lib
    rng = np.random.default_rng(9)
    hq, hkv, d, n = 4, 1, 128, 300
    for power, spread in ((126.0, 1.0), (-95.0, 1.0), (0.0, 300.0)):
        x = bf16_to_f64(rand_bf16(rng, (2, 19, hkv, BS, d)))
        x = np.clip(x, -3.9, 3.9)
        slabs = Q.blocks(x[0] * spread, np.clip(x[1], -1.9, 1.9) * 2.0**power, d, bits)
        tables = rng.permutation(19)[None].astype(np.int32)
        q = rand_bf16(rng, (1, hq, d))
        out = torch.empty((1, hq, d), dtype=torch.bfloat16, device="cuda")
        lib.pkv_quant_decode_attention(torch.from_numpy(slabs).cuda(), to_dev_bits(q), i32(tables), i32([n]), n, 0.09,
                                       out)
        k, v = sequence(slabs, tables[0], n, d, bits)
        o, _, tol, _ = rows_of(bf16_to_f64(q[0]), k[0], v[0], 0.09, 2.0**-16)
        got = bf16_to_f64(to_host_bits(out))[0]
        assert np.isfinite(got).all() and (np.abs(got - o) <= tol + 2.0**-126).all(), (power, spread)


def parts_off(q, bits):
    """What three parts of e2m3 leave of queries beside 4-bit keys. With the largest of 32 in [4, 8): codes have steps
    of 1/8 below 2 and 4 bits above, parts are 2^-4 of each other, so what is left is a multiple of 2^-11 or less than
    half of that. A bf16 of 2^-4 and more, which is 2^-6 of the largest at least (less 2^-7 of itself), is a multiple."""
    if bits == 8:
        return 0.0
    x = np.abs(q).reshape(*q.shape[:-1], -1, 32)
    top = x.max(-1, keepdims=True)
    return np.where(x < 2.0**-6 * top, 2.0**-14 * top, 0.0).reshape(q.shape)


def check_prefill(lib, rng, cached, new, hq, hkv, d, bits, split=True):
    import torch
    cached, new = np.array(cached), np.array(new)
    lens = cached + new
    tables, host = pool(rng, lens.tolist(), hkv, d, bits)
    t, b = int(new.sum()), len(new)
    cache = torch.from_numpy(host).cuda()
    q = rand_bf16(rng, (t, hq, d))
    scale = 1 / math.sqrt(d)
    cu = np.concatenate([[0], np.cumsum(new)])
    need = lib.pkv_quant_prefill_workspace_bytes(b, t, hq, hkv, d, bits, int(new.max()), int(lens.max()))
    ws = torch.full((need + 64,), 255, dtype=torch.uint8, device="cuda") if split and need else None
    out = torch.full((t + 1, hq, d), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((t + 1, hq), 7.0, device="cuda")
    lib.pkv_quant_prefill_attention(cache, to_dev_bits(q), i32(tables), i32(cached), i32(cu), int(new.max()),
                                    int(lens.max()), scale, out[:t], lse=lse[:t],
                                    workspace=None if ws is None else ws[:need])
    torch.cuda.synchronize()
    assert (out[t] == 7).all() and (lse[t] == 7).all() and (ws is None or (ws[need:] == 255).all())
    got, got_lse = bf16_to_f64(to_host_bits(out[:t])), lse[:t].double().cpu().numpy()
    assert np.isfinite(got).all() and np.isfinite(got_lse).all()
    g, worst = hq // hkv, 0.0
    for i in range(b):
        if new[i] == 0:
            continue
        k, v = sequence(host, tables[i], int(lens[i]), d, bits)
        for j in sorted({0, int(new[i]) // 2, int(new[i]) - 1}):
            n, row = int(cached[i]) + j + 1, cu[i] + j
            for h in range(hkv):
                rows = slice(h * g, h * g + g)
                x = bf16_to_f64(q[row, rows])
                o, z, tol, tol_z = rows_of(x, k[h, :n], v[h, :n], scale, 2.0**-8, parts_off(x, bits))
                err = np.abs(got[row, rows] - o)
                assert (err <= tol).all(), (i, j, h, float((err / tol).max()))
                assert (np.abs(got_lse[row, rows] - z) <= tol_z).all(), (i, j, h)
                worst = max(worst, float((err / np.maximum(tol, 1e-300)).max()))
    say(f"  prefill {hq}/{hkv} heads of {d}, bits {bits}: {worst:.2f} of the tolerance")


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("hq,hkv,d", [(4, 2, 64), (8, 2, 128), (3, 3, 128), (20, 1, 64)])
def test_prefill(gpu_lib, hq, hkv, d, bits):
    rng = np.random.default_rng(hq + d + bits)
    say(f"[quant prefill] {hq}/{hkv} heads of {d}, bits {bits}")
    check_prefill(gpu_lib, rng, [0, 5, 16, 63, 64, 130, 100, 0, 250], [1, 3, 0, 1, 64, 37, 200, 70, 2], hq, hkv, d, bits)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("split", [False, True])
def test_prefill_long(gpu_lib, bits, d, split):
    """Splits of 1024 keys and more, ordered batches."""
    rng = np.random.default_rng(d + bits)
    say(f"[quant prefill] long, heads of {d}, bits {bits}, split {split}")
    check_prefill(gpu_lib, rng, [4000, 1000, 2500], [33, 70, 1], 4, 2, d, bits, split)
    check_prefill(gpu_lib, rng, [8300, 10, 1500] + [7] * 20, [9, 70, 1] + [5] * 20, 4, 1, d, bits, split)


def test_prefill_many_items(gpu_lib):
    rng = np.random.default_rng(10)
    for bits, (hq, hkv, d) in ((4, (32, 8, 128)), (8, (16, 4, 64)), (8, (32, 8, 128)), (4, (64, 8, 128))):
        check_prefill(gpu_lib, rng, rng.integers(0, 900, 24), rng.integers(0, 150, 24), hq, hkv, d, bits)


@pytest.mark.parametrize("bits", [4, 8])
def test_prefill_plans(gpu_lib, bits):
    """The sides of the plan: a few items cut to fill the chip, cuts of 3008 keys behind an ordering launch, items that
    fill the chip in order, and one sequence alone; lengths of none and one among them."""
    rng = np.random.default_rng(20 + bits)
    lib = gpu_lib
    sizes = lambda b, *a: lib.pkv_quant_prefill_workspace_bytes(b, *a)
    check_prefill(lib, rng, [3000], [64], 8, 2, 64, bits)
    check_prefill(lib, rng, rng.integers(0, 700, 17).tolist() + [3900, 0], [1, 0] + rng.integers(1, 9, 17).tolist(), 8, 8,
                  64, bits)
    assert sizes(19, 90, 8, 8, 64, bits, 8, 3908) > 90 * 8 * 2 * 66 * 4  # (split in two)
    cached, new = rng.integers(0, 300, 20), rng.integers(60, 140, 20)
    cached[3] = 2500
    check_prefill(lib, rng, cached, new, 32, 8, 64, bits)
    assert 0 < sizes(20, int(new.sum()), 32, 8, 64, bits, int(new.max()), 2640) < 4096  # (an order alone)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("d", [64, 128])
def test_prefill_nan_reaches_the_rows_that_see_it(gpu_lib, bits, d):
    """A token that reads back as NaN, key or value: rows before it keep their bits, rows from it on are NaN, and so
    no head of another kv head."""
    import torch
    lib = gpu_lib
    rng = np.random.default_rng(bits + d)
    hq, hkv, cached, new = 4, 2, 300, 200
    n = cached + new
    tables, clean = pool(rng, [n], hkv, d, bits)
    q = to_dev_bits(rand_bf16(rng, (new, hq, d)))
    args = i32(tables), i32([cached]), i32([0, new]), new, n, 0.1
    out = torch.empty((new, hq, d), dtype=torch.bfloat16, device="cuda")
    lib.pkv_quant_prefill_attention(torch.from_numpy(clean).cuda(), q, *args, out)
    assert torch.isfinite(out).all()
    for part in (1, 3):  # key scales, value scales
        for at in (cached + 70, n - 1, 5):
            cache = clean.copy()
            parts = [x.copy() for x in Q.parts(cache[tables[0, at // BS]], d, bits)]
            parts[part][1, at % BS] = 255 if part == 1 else np.nan
            cache[tables[0, at // BS]] = Q.joined(*parts, d, bits)
            hurt = torch.empty_like(out)
            lib.pkv_quant_prefill_attention(torch.from_numpy(cache).cuda(), q, *args, hurt)
            first = max(at - cached, 0)
            assert torch.isnan(hurt[first:, 2:]).all(), (part, at)
            hurt[first:, 2:] = out[first:, 2:]
            assert torch.equal(hurt.view(torch.int16), out.view(torch.int16)), (part, at)


def test_prefill_queries_that_are_not_finite(gpu_lib):
    import torch
    lib = gpu_lib
    rng = np.random.default_rng(8)
    hq, hkv, d, bits, cached, new = 8, 2, 64, 4, 100, 90
    tables, cache = pool(rng, [cached + new], hkv, d, bits)
    q = rand_bf16(rng, (new, hq, d))
    q[3, 1, 5], q[80, 6, 7] = 0x7F80, 0x7FC0
    out = torch.empty((new, hq, d), dtype=torch.bfloat16, device="cuda")
    lib.pkv_quant_prefill_attention(torch.from_numpy(cache).cuda(), to_dev_bits(q), i32(tables), i32([cached]),
                                    i32([0, new]), new, cached + new, 0.1, out)
    bad = torch.isnan(out).any(2).cpu().numpy()
    assert bad[3, 1] and bad[80, 6] and bad.sum() == 2


@pytest.mark.parametrize("bits", [4, 8])
def test_prefill_extreme_scales(gpu_lib, bits):
    """Values near the largest and the least, and scores far apart: no sum leaves the 32-bit range. (A weight times
    a scale near 2^-98 may lose the bits below 2^-133, the least bf16: 300 keys' codes of 448 at most, which is less
    than 2^-115.)"""
    import torch
    lib = gpu_lib
    rng = np.random.default_rng(9)
    hq, hkv, d, n, new = 4, 1, 128, 300, 40
    for power, spread in ((126.0, 1.0), (-95.0, 1.0), (0.0, 300.0)):
        x = np.clip(bf16_to_f64(rand_bf16(rng, (2, 19, hkv, BS, d))), -3.9, 3.9)
        slabs = Q.blocks(x[0] * spread, np.clip(x[1], -1.9, 1.9) * 2.0**power, d, bits)
        tables = rng.permutation(19)[None].astype(np.int32)
        q = rand_bf16(rng, (new, hq, d))
        out = torch.empty((new, hq, d), dtype=torch.bfloat16, device="cuda")
        lib.pkv_quant_prefill_attention(torch.from_numpy(slabs).cuda(), to_dev_bits(q), i32(tables), i32([n - new]),
                                        i32([0, new]), new, n, 0.09, out)
        got = bf16_to_f64(to_host_bits(out))
        k, v = (y.copy() for y in sequence(slabs, tables[0], n, d, bits))
        for j in (0, new // 2, new - 1):
            at = n - new + j + 1
            y = bf16_to_f64(q[j])
            o, _, tol, _ = rows_of(y, k[0, :at], v[0, :at], 0.09, 2.0**-8, parts_off(y, bits))
            assert np.isfinite(got[j]).all() and (np.abs(got[j] - o) <= tol + 2.0**-115).all(), (power, spread, j)
