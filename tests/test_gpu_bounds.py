"""GPU tier: key bounds per block (pkv_block_bounds) against a loop over blocks. A bound is one of
its keys' own values, so everything is compared exactly; blocks without new tokens, and blocks
past a sequence's end, keep every bit."""
import numpy as np
import pytest

from tests.gpu_util import bf16_to_f64, i32, say, to_dev_bits, to_host_bits
from tests.paged_fixture import rand_bf16

pytestmark = pytest.mark.gpu

BS = 16
NAN = 0x7FC0


def case(rng, seqs, hkv, d, width=None):
    """Pool, tables and stale bounds; slots past a sequence's end hold NaN."""
    blocks = [-(-(c + n) // BS) for c, n in seqs]
    nb = sum(blocks) + 2
    perm = rng.permutation(nb)
    width = width or max(blocks) + 1
    tables = np.full((len(seqs), width), -1, np.int32)
    pk = rand_bf16(rng, (nb, hkv, d // 8, BS, 8))
    at = 0
    for i, b in enumerate(blocks):
        b = min(b, width)
        tables[i, :b] = perm[at:at + b]
        at += b
        tail = sum(seqs[i]) % BS
        if tail and b == blocks[i]:
            pk[tables[i, b - 1], :, :, tail:] = NAN
    return pk, tables, rand_bf16(rng, (nb, hkv, 2, d))


def call(lib, pk, tables, bounds, seqs, max_new=None, stream=None):
    import torch
    nb, hkv, nch = pk.shape[:3]
    kc, out = to_dev_bits(pk), to_dev_bits(bounds)
    vc = torch.zeros((nb, hkv, nch * 8, BS), dtype=torch.bfloat16, device="cuda")
    cu = np.concatenate([[0], np.cumsum([n for _, n in seqs])])
    lib.pkv_block_bounds(kc, vc, out, i32(tables), i32([c for c, _ in seqs]), i32(cu),
                         max_new or max(n for _, n in seqs), stream=stream)
    torch.cuda.synchronize()
    return to_host_bits(out)


def expect(pk, tables, bounds, seqs):
    nb, hkv, nch = pk.shape[:3]
    want = bf16_to_f64(bounds)
    touched = np.zeros(nb, bool)
    for i, (c, n) in enumerate(seqs):
        if n == 0:
            continue
        for b in range(c // BS, min(-(-(c + n) // BS), tables.shape[1])):
            blk = tables[i, b]
            keys = bf16_to_f64(pk[blk, :, :, :min(BS, c + n - b * BS)])  # [hkv, nch, s, 8]
            want[blk, :, 0] = keys.max(2).reshape(hkv, nch * 8)  # (a NaN propagates)
            want[blk, :, 1] = keys.min(2).reshape(hkv, nch * 8)
            touched[blk] = True
    return want, touched


def check(got, pk, tables, bounds, seqs):
    want, touched = expect(pk, tables, bounds, seqs)
    assert np.array_equal(bf16_to_f64(got)[touched], want[touched], equal_nan=True)
    assert np.array_equal(got[~touched], bounds[~touched]), "untouched blocks"


SEQS = [(0, 1), (15, 1), (16, 1), (0, 16), (3, 40), (33, 0), (100, 200), (31, 2), (17, 31)]


@pytest.mark.parametrize("hkv,d", [(1, 64), (2, 128), (5, 64), (8, 128), (20, 128)])
@pytest.mark.parametrize("seqs", [SEQS[:1], SEQS, [(i * 7, 1) for i in range(50)], [(5, 4000)]])
def test_matches_a_loop_over_blocks(gpu_lib, hkv, d, seqs):
    say(f"[bounds] {len(seqs)} sequences, {hkv} heads of {d}")
    rng = np.random.default_rng(d + hkv)
    args = case(rng, seqs, hkv, d)
    check(call(gpu_lib, *args, seqs), *args, seqs)
    check(call(gpu_lib, *args, seqs, max_new=5000), *args, seqs)
    check(call(gpu_lib, *args, seqs, max_new=1 << 24), *args, seqs)  # (as keys past the caches)


def test_special_values(gpu_lib):
    """Infinities are ordinary bounds, a NaN of a live key makes both bounds NaN, equal keys
    give equal bounds, and the zeros' signs do not matter."""
    rng = np.random.default_rng(2)
    seqs = [(0, 16), (0, 9), (0, 4), (0, 16)]
    pk, tables, bounds = case(rng, seqs, 2, 64)
    pk[tables[0, 0], 0, 0, 5] = 0x7F80   # +inf
    pk[tables[0, 0], 1, 3, 9] = 0xFF80   # -inf
    pk[tables[0, 0], 0, 2, 0, 3] = NAN
    pk[tables[1, 0], 1, 1, 8, 2] = 0xFFC1  # a NaN with its sign set, in the last live slot
    pk[tables[2, 0], :, :, :4] = 0x3F80
    pk[tables[3, 0], :, 0, ::2] = 0x8000
    pk[tables[3, 0], :, 0, 1::2] = 0
    got = call(gpu_lib, pk, tables, bounds, seqs)
    check(got, pk, tables, bounds, seqs)
    v = bf16_to_f64(got)
    assert np.isnan(v[tables[0, 0], 0, :, 19]).all() and np.isnan(v[tables[1, 0], 1, :, 10]).all()
    assert np.isnan(v).sum() == np.isnan(bf16_to_f64(bounds)).sum() + 4


def test_ids_outside_the_pool_and_past_the_table_are_skipped(gpu_lib):
    rng = np.random.default_rng(3)
    seqs = [(0, 100), (0, 40)]
    pk, tables, bounds = case(rng, seqs, 2, 128, width=3)
    tables[1, 1] = -1
    tables[1, 2] = len(pk)
    got = call(gpu_lib, pk, tables, bounds, seqs)
    check(got, pk, tables[:, :3], bounds, [(0, 48), (0, 16)])


def test_another_stream_and_a_replay(gpu_lib):
    import torch
    lib = gpu_lib
    rng = np.random.default_rng(4)
    pk, tables, bounds = case(rng, SEQS, 2, 128)
    side = torch.cuda.Stream()
    check(call(lib, pk, tables, bounds, SEQS, stream=side), pk, tables, bounds, SEQS)
    kc, out = to_dev_bits(pk), to_dev_bits(bounds)
    vc = torch.zeros((len(pk), 2, 128, BS), dtype=torch.bfloat16, device="cuda")
    args = (i32(tables), i32([c for c, _ in SEQS]),
            i32(np.concatenate([[0], np.cumsum([n for _, n in SEQS])])), 200)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            lib.pkv_block_bounds(kc, vc, out, *args)
    for _ in range(3):
        pk, _, _ = case(rng, SEQS, 2, 128)
        pk = rand_bf16(rng, pk.shape)
        kc.copy_(to_dev_bits(pk))
        graph.replay()
        torch.cuda.synchronize()
        check(to_host_bits(out), pk, tables, bounds, SEQS)
