"""GPU tier, bit-exact: the quantised cache's append and its conversions from and to the bf16 pool against the
oracle. Whole pools are compared, so a stray write anywhere fails the test; what holds no token starts as
bytes of 255 (NaN throughout) in the cache and as NaN in the bf16 pool."""
import numpy as np
import pytest

from oracle import quant as Q
from tests.gpu_util import bf16_to_f64, i32, say, to_dev_bits, to_host_bits
from tests.paged_fixture import rand_bf16

pytestmark = pytest.mark.gpu

BS = 16
INF, NEG_INF, NAN, BIG, TINY, LEAST = 0x7F80, 0xFF80, 0x7FC0, 0x7F7F, 0x0D80, 0x0001


def rows(rng, n, hkv, d, special=False):
    """bf16 bits [n][hkv][d] over many magnitudes; with zeros of both signs, and special values here and
    there."""
    x = rand_bf16(rng, (n, hkv, d))
    step = rng.integers(-9, 9, (n, hkv, 1)).astype(np.int64)
    x = (x.astype(np.int64) + (step << 7)).astype(np.uint16)  # (times powers of two)
    x[rng.random(x.shape) < 0.05] = 0x8000
    if special:
        for value in (INF, NEG_INF, NAN, BIG, BIG | 0x8000, TINY, TINY - 1, LEAST, 0):
            x[rng.integers(0, n), rng.integers(0, hkv), rng.integers(0, d)] = value
        x[rng.integers(0, n), rng.integers(0, hkv)] = 0
        x[rng.integers(0, n), rng.integers(0, hkv)] = LEAST
        x[rng.integers(0, n), rng.integers(0, hkv)] = TINY
        x[rng.integers(0, n), rng.integers(0, hkv)] = 0x7F00 | rng.integers(0, 128, d).astype(np.uint16)
    return x


def borders(rng, n, hkv, d, bits):
    """Rows of values on the borders between codes, with a largest value that gives a known scale."""
    v = np.unique(np.abs(Q.code_values(bits)[~np.isnan(Q.code_values(bits))]))
    mid = (v[:-1] + v[1:]) / 2
    x = rng.choice(np.concatenate([mid, v]), (n, hkv, d)) * rng.choice([-1.0, 1.0], (n, hkv, d))
    x[..., ::32] = Q.MOST[bits]
    m = rng.integers(8, 16, (n, 1, 1))  # scales of 4 bits (exact products: 5 bits by 4)
    x = x * m * 2.0 ** rng.integers(-20, 20, (n, 1, 1))
    return (x.astype(np.float32).view(np.uint32) >> 16).astype(np.uint16)


def pool_of(lens_after, rng, extra=3):
    counts = [-(-n // BS) for n in lens_after]
    nb = sum(counts) + extra
    perm = rng.permutation(nb)
    tables = np.full((len(counts), max(counts) + 1), -1, np.int32)
    at = 0
    for i, c in enumerate(counts):
        tables[i, :c] = perm[at:at + c]
        at += c
    return tables, nb


def places(tables, cached, new):
    return [(tables[i, p // BS], p % BS) for i in range(len(new)) for p in range(cached[i], cached[i] + new[i])]


def same_bytes(got, ref):
    got = got.cpu().numpy()
    bad = np.argwhere(got != ref)
    assert not len(bad), f"{len(bad)} bytes differ, first at {bad[0]}: {got[tuple(bad[0])]} not {ref[tuple(bad[0])]}"


HEADS = [(1, 128), (2, 64), (3, 64), (5, 128), (8, 128)]


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("hkv,d", HEADS)
def test_append(gpu_lib, bits, hkv, d):
    """Ragged ranges that begin and end anywhere in a block, empty ones among them, in one call; then one
    token a sequence, in several steps, into what the first call left."""
    import torch
    lib = gpu_lib
    say(f"[quant append] bits {bits}, {hkv} heads of {d}")
    rng = np.random.default_rng(100 * bits + d + hkv)
    cached = np.array([0, 5, 16, 17, 31, 40, 100, 7, 3])
    new = np.array([3, 0, 16, 1, 40, 0, 77, 9, 2])
    tables, nb = pool_of(cached + new + 4, rng)
    ref = np.full((nb, hkv, Q.slab_bytes(d, bits)), 255, np.uint8)
    cache = torch.from_numpy(ref).cuda()
    for step in range(4):
        t = int(new.sum())
        k, v = (rows(rng, t, hkv, d, special=step == 1) for _ in range(2))
        # parts of wider rows
        wide = np.full((t, 2 * hkv + 1, d), NAN, np.uint16)
        wide[:, :hkv], wide[:, hkv + 1:] = k, v
        dev = to_dev_bits(wide)
        lib.pkv_quant_append(cache, dev[:, :hkv], dev[:, hkv + 1:], i32(tables), i32(cached),
                             i32(np.concatenate([[0], np.cumsum(new)])), int(new.max()))
        torch.cuda.synchronize()
        ref = Q.written(ref, places(tables, cached, new), bf16_to_f64(k), bf16_to_f64(v), d, bits)
        same_bytes(cache, ref)
        cached = cached + new
        new = np.minimum(1, rng.integers(0, 4, len(cached))) if step else np.ones(len(cached), np.int64)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("d", [64, 128])
def test_append_special_values(gpu_lib, bits, d):
    import torch
    lib = gpu_lib
    say(f"[quant append] special values, bits {bits}, d {d}")
    rng = np.random.default_rng(7 * bits + d)
    for seed in range(4):
        n = 61
        tables, nb = pool_of([n + 5], rng)
        k, v = rows(rng, n, 2, d, special=True), rows(rng, n, 2, d, special=True)
        if seed >= 2:
            k, v = borders(rng, n, 2, d, bits), borders(rng, n, 2, d, bits)
        ref = np.full((nb, 2, Q.slab_bytes(d, bits)), 255, np.uint8)
        cache = torch.from_numpy(ref).cuda()
        lib.pkv_quant_append(cache, to_dev_bits(k), to_dev_bits(v), i32(tables), i32([5]), i32([0, n]), n)
        torch.cuda.synchronize()
        same_bytes(cache, Q.written(ref, places(tables, [5], [n]), bf16_to_f64(k), bf16_to_f64(v), d, bits))


@pytest.mark.parametrize("bits", [4, 8])
def test_append_bad_metadata_stays_in_bounds(gpu_lib, bits):
    """Table entries outside the pool, positions past the table, rows past the last: skipped, or zeros."""
    import torch
    lib = gpu_lib
    rng = np.random.default_rng(bits)
    hkv, d, nb = 2, 64, 4
    ref = np.full((nb, hkv, Q.slab_bytes(d, bits)), 255, np.uint8)
    cache = torch.from_numpy(ref).cuda()
    k, v = rows(rng, 20, hkv, d), rows(rng, 20, hkv, d)
    tables = np.array([[-1, 4], [99, 1], [2, 0]], np.int32)
    lib.pkv_quant_append(cache, to_dev_bits(k), to_dev_bits(v), i32(tables), i32([0, 30, 31]), i32([0, 18, 20, 24]),
                         18)
    torch.cuda.synchronize()
    kf, vf = bf16_to_f64(k), bf16_to_f64(v)
    # sequence 1: slots 14, 15 of block 1; sequence 2: slot 15 of block 0, a row past the end
    ref = Q.written(ref, [(1, 14), (1, 15), (0, 15)], np.concatenate([kf[18:20], 0 * kf[:1]]),
                    np.concatenate([vf[18:20], 0 * vf[:1]]), d, bits)
    same_bytes(cache, ref)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("hkv,d", HEADS)
def test_blocks_there_and_back(gpu_lib, bits, hkv, d):
    import torch
    lib = gpu_lib
    say(f"[quant blocks] bits {bits}, {hkv} heads of {d}")
    rng = np.random.default_rng(bits + d + hkv)
    nb, nq = 23, 17
    k, v = (rows(rng, nb * BS, hkv, d, special=True).reshape(nb, BS, hkv, d) for _ in range(2))
    k[3], v[4] = NAN, INF
    k[5:7] = borders(rng, 2 * BS, hkv, d, bits).reshape(2, BS, hkv, d)
    v[5:7] = borders(rng, 2 * BS, hkv, d, bits).reshape(2, BS, hkv, d)
    pk = k.transpose(0, 2, 3, 1).reshape(nb, hkv, d // 8, 8, BS).transpose(0, 1, 2, 4, 3).copy()
    pv = v.transpose(0, 2, 3, 1).copy()
    pairs = np.stack([rng.permutation(nb)[:nq - 2], rng.permutation(nq)[:nq - 2]], 1)
    bad = np.array([[-1, 0], [0, -1], [nb, 1], [1, nq], [2**31 - 1, -2**31]])
    ref = np.full((nq, hkv, Q.slab_bytes(d, bits)), 255, np.uint8)
    cache = torch.from_numpy(ref).cuda()
    dk, dv = to_dev_bits(pk), to_dev_bits(pv)
    lib.pkv_quant_blocks(dk, dv, cache, i32(np.concatenate([pairs, bad])))
    torch.cuda.synchronize()
    slabs = Q.blocks(bf16_to_f64(k).transpose(0, 2, 1, 3), bf16_to_f64(v).transpose(0, 2, 1, 3), d, bits)
    ref[pairs[:, 1]] = slabs[pairs[:, 0]]
    same_bytes(cache, ref)
    assert np.array_equal(to_host_bits(dk), pk) and np.array_equal(to_host_bits(dv), pv)

    # back, into other blocks of a pool of ones
    back = np.stack([rng.permutation(nq)[:9], rng.permutation(nb)[:9]], 1)
    bad = np.array([[-1, 0], [0, nb], [nq, 1]])
    ok, ov = np.full_like(pk, 0x3F80), np.full_like(pv, 0x3F80)
    dk, dv = to_dev_bits(ok), to_dev_bits(ov)
    lib.pkv_dequant_blocks(cache, dk, dv, i32(np.concatenate([back, bad])))
    torch.cuda.synchronize()
    same_bytes(cache, ref)
    ek, ev = Q.stands_for(ref, d, bits)  # [nq][hkv][16][d]
    gk, gv = bf16_to_f64(to_host_bits(dk)), bf16_to_f64(to_host_bits(dv))
    rest = np.setdiff1d(np.arange(nb), back[:, 1])
    assert (gk[rest] == 1).all() and (gv[rest] == 1).all()
    gk = gk[back[:, 1]].transpose(0, 1, 3, 2, 4).reshape(9, hkv, BS, d)
    gv = gv[back[:, 1]].transpose(0, 1, 3, 2)
    for got, want in ((gk, ek[back[:, 0]]), (gv, ev[back[:, 0]])):
        assert np.array_equal(got, want, equal_nan=True)
        fine = ~np.isnan(want)
        assert np.array_equal(np.signbit(got[fine]), np.signbit(want[fine]))


def test_append_is_what_the_blocks_call_writes(gpu_lib):
    """Whole blocks of rows, appended to either pool: the same cache."""
    import torch
    lib = gpu_lib
    rng = np.random.default_rng(5)
    hkv, d, n = 4, 128, 160
    tables, nb = pool_of([n], rng)
    k, v = to_dev_bits(rows(rng, n, hkv, d)), to_dev_bits(rows(rng, n, hkv, d))
    pk = torch.zeros((nb, hkv, d // 8, BS, 8), dtype=torch.bfloat16, device="cuda")
    pv = torch.zeros((nb, hkv, d, BS), dtype=torch.bfloat16, device="cuda")
    args = i32(tables), i32([0]), i32([0, n]), n
    lib.pkv_kv_append(pk, pv, k, v, *args)
    pairs = i32(np.stack([tables[0, :n // BS]] * 2, 1))
    for bits in (4, 8):
        a, b = (lib.alloc_quant_cache(nb, hkv, d, bits).fill_(9) for _ in range(2))
        lib.pkv_quant_append(a, k, v, *args)
        lib.pkv_quant_blocks(pk, pv, b, pairs)
        assert torch.equal(a, b)


def test_offsets_past_32_bits(gpu_lib):
    """Blocks whose bytes lie behind 2^32, in both pools, and rows behind 2^31 elements."""
    import torch
    lib = gpu_lib
    rng = np.random.default_rng(6)
    hkv, d, bits = 8, 128, 8
    nb = (1 << 32) // (hkv * Q.slab_bytes(d, bits)) + 9
    say(f"[quant blocks] {nb} blocks")
    cache = lib.alloc_quant_cache(nb, hkv, d, bits)
    pk = torch.empty((nb, hkv, d // 8, BS, 8), dtype=torch.bfloat16, device="cuda")
    pv = torch.empty((nb, hkv, d, BS), dtype=torch.bfloat16, device="cuda")
    k, v = rows(rng, 2 * BS, hkv, d), rows(rng, 2 * BS, hkv, d)
    far = torch.zeros((1 << 31) + 2 * BS * hkv * d, dtype=torch.bfloat16, device="cuda")
    wide = far.as_strided((2 * BS, hkv, d), ((1 << 31) // (2 * BS - 1) // 8 * 8, d, 1))
    wide.copy_(to_dev_bits(k))
    last = np.array([nb - 1, nb - 2])
    tables = np.array([last], np.int32)
    lib.pkv_quant_append(cache, wide, to_dev_bits(v), i32(tables), i32([0]), i32([0, 2 * BS]), 2 * BS)
    ref = Q.blocks(*(bf16_to_f64(x).reshape(2, BS, hkv, d).transpose(0, 2, 1, 3) for x in (k, v)), d, bits)
    same_bytes(cache[last], ref)
    lib.pkv_dequant_blocks(cache, pk, pv, i32(np.stack([last, last - 2], 1)))
    lib.pkv_quant_blocks(pk, pv, cache, i32(np.stack([last - 2, last - 4], 1)))
    torch.cuda.synchronize()
    ek, ev = Q.stands_for(ref, d, bits)
    got = bf16_to_f64(to_host_bits(pv[last - 2])).transpose(0, 1, 3, 2)
    assert np.array_equal(got, ev)
    k2, v2 = Q.stands_for(cache[last - 4].cpu().numpy(), d, bits)
    assert np.array_equal(k2, ek)  # (keys come back as they are: a power of two more or less changes none)
    assert np.abs(v2 - ev).max() <= 2.0**-3 * np.abs(ev).max()
