"""GPU tier: the choice of blocks (pkv_select_blocks) against its definition in 64 bits. A choice
has no tolerance: the chosen blocks must be the same, also where scores differ by less than 32-bit
sums can tell, where they are equal, and where they are not finite."""
import math

import numpy as np
import pytest

from tests.gpu_util import bf16_to_f64, i32, say, to_dev_bits
from tests.paged_fixture import rand_bf16

pytestmark = pytest.mark.gpu

BS = 16


def bf16(x):
    """float values that bf16 holds, as bits"""
    u = np.asarray(x, np.float32).view(np.uint32)
    assert not (u & 0xFFFF).any()
    return (u >> 16).astype(np.uint16)


def choice(bounds, q, table, length, sink, recent, blocks):
    """One row's blocks per kv head: bounds, q as float64."""
    hkv = bounds.shape[1]
    g = q.shape[0] // hkv
    n = min(-(-length // BS), len(table)) if length > 0 else 0
    out = np.full((hkv, blocks), -1, np.int64)
    for h in range(hkv):
        box = bounds[table[:n], h]                                    # [n, 2, d]
        qh = q[h * g:(h + 1) * g, None]                               # [g, 1, d]
        with np.errstate(invalid="ignore", over="ignore"):
            s = np.where(qh > 0, qh * box[:, 0], qh * box[:, 1]).sum(2)
            # whatever is not finite in a row's queries or a block's bounds makes it first
            s = np.where(np.isfinite(qh).all(2) & np.isfinite(box).all((1, 2)), s, math.inf)
        s = np.where(np.isfinite(s), s, math.inf).max(0) if n else np.zeros(0)
        taken = [b for b in range(n) if b < sink or b >= n - recent]
        rest = sorted((b for b in range(n) if sink <= b < n - recent), key=lambda b: (-s[b], b))
        got = sorted((taken + rest)[:blocks])
        out[h, :len(got)] = got
    return out


def pool(rng, lens, hkv, d, nan=True):
    """Tables in random order and bounds about their keys; blocks of no sequence hold NaN."""
    counts = [-(-n // BS) for n in lens]
    nb = sum(counts) + 3
    perm = rng.permutation(nb)
    tables = np.full((len(lens), max(counts) + 1), -1, np.int32)
    at = 0
    for i, c in enumerate(counts):
        tables[i, :c] = perm[at:at + c]
        at += c
    mid, reach = rng.standard_normal((2, nb, hkv, 1, d))
    box = np.concatenate([mid + abs(reach), mid - abs(reach)], axis=2).astype(np.float32)
    bits = (box.view(np.uint32) >> 16).astype(np.uint16)
    if nan:
        bits[perm[at:]] = 0x7FC0
    return tables, bits


def run(lib, tables, bounds, q, row_lens, sink, recent, blocks, row_seq=None, max_len=None,
        stream=None):
    import torch
    t, hkv = len(q), bounds.shape[1]
    sel = torch.full((t, hkv, blocks), -7, dtype=torch.int32, device="cuda")
    lib.pkv_select_blocks(to_dev_bits(bounds), to_dev_bits(q), i32(tables), i32(row_lens),
                          max_len or max(1, int(np.max(row_lens))), sink, recent, sel,
                          row_seq=None if row_seq is None else i32(row_seq), stream=stream)
    torch.cuda.synchronize()
    return sel.cpu().numpy()


def check(got, tables, bounds, q, row_lens, sink, recent, blocks, row_seq=None, max_len=None):
    b64, q64 = bf16_to_f64(bounds), bf16_to_f64(q)
    for t in range(len(q)):
        s = t if row_seq is None else row_seq[t]
        if s < 0:
            assert (got[t] == -7).all(), "a padding row was written"
            continue
        n = min(row_lens[t], max_len or row_lens[t])
        want = choice(b64, q64[t], tables[s], n, sink, recent, blocks)
        assert np.array_equal(got[t], want), (t, n, np.argwhere(got[t] != want)[:4])


HEADS = [(4, 2, 64), (32, 8, 128), (8, 8, 64), (16, 1, 128), (28, 4, 128), (3, 1, 64)]


@pytest.mark.parametrize("hq,hkv,d", HEADS)
@pytest.mark.parametrize("lens,sink,recent,blocks", [
    ([1, 15, 16, 17, 5], 0, 1, 1),
    ([400, 129, 128, 127, 2000], 1, 2, 8),
    ([5000, 33, 777], 3, 5, 8),
    ([5000, 33, 777], 0, 1, 200),
    ([16 * 129, 16 * 128, 16 * 127], 2, 2, 128),
    ([16 * 64, 16 * 63 + 1, 700], 1, 2, 20),     # (up to 64 blocks: a wave each)
    ([16 * 64 + 1, 30, 900], 0, 2, 20),
    ([16 * 512, 16 * 511 + 3, 16 * 257], 2, 1, 100),  # (up to 512: one launch)
    ([16 * 512 + 1, 100, 16 * 400], 2, 1, 100),
])
def test_decode_rows(gpu_lib, hq, hkv, d, lens, sink, recent, blocks):
    say(f"[select] {hq}/{hkv} heads of {d}, {lens}, {sink}+{recent} of {blocks}")
    rng = np.random.default_rng(d + hq)
    tables, bounds = pool(rng, lens, hkv, d)
    q = rand_bf16(rng, (len(lens), hq, d))
    args = (tables, bounds, q, np.array(lens), sink, recent, blocks)
    check(run(gpu_lib, *args), *args)


@pytest.mark.parametrize("hq,hkv,d", HEADS)
def test_rows_of_longer_suffixes(gpu_lib, hq, hkv, d):
    """Rows of several sequences, of none (padding), without keys, and past the host's length."""
    rng = np.random.default_rng(hq)
    lens = [900, 40, 1500]
    tables, bounds = pool(rng, lens, hkv, d)
    seq, seen = [], []
    for s, n in ((0, 37), (1, 9), (2, 50)):
        seq += [s] * n
        seen += list(range(lens[s] - n + 1, lens[s] + 1))
    seq[3] = seq[20] = seq[60] = -1
    seen[5] = seen[70] = 0
    seen[6], seen[71] = 1, 200
    q = rand_bf16(rng, (len(seq), hq, d))
    args = (tables, bounds, q, np.array(seen), 1, 2, 9, np.array(seq))
    check(run(gpu_lib, *args), *args)
    check(run(gpu_lib, *args, max_len=640), *args, max_len=640)
    mixed = rng.permutation(len(seq))
    args = (tables, bounds, q, np.array(seen)[mixed], 1, 2, 9, np.array(seq)[mixed])
    check(run(gpu_lib, *args), *args)


def test_long_rows(gpu_lib):
    rng = np.random.default_rng(8)
    lens = [16 * 30000 + 5, 16 * 8192, 16 * 8193, 1 << 20]
    tables, bounds = pool(rng, lens, 1, 64)
    q = rand_bf16(rng, (len(lens), 2, 64))
    args = (tables, bounds, q, np.array(lens), 1, 4, 700)
    check(run(gpu_lib, *args), *args)


@pytest.mark.parametrize("n", [40, 300, 600, 2000])
def test_scores_that_32_bits_cannot_tell_apart(gpu_lib, n):
    """Sums near 2^10 that differ by 2^-20 and less, in random order: all of them candidates."""
    rng = np.random.default_rng(n)
    hq, hkv, d = 4, 2, 128
    tables, bounds = pool(rng, [n * BS], hkv, d)
    base = bf16(rng.integers(1, 128, (hkv, 1, d)) / 8.0)
    bounds[tables[0, :n]] = base
    step = rng.permutation(n).reshape(n, 1)  # two dims carry a number of 14 bits, in units of 2^-30
    bounds[tables[0, :n], :, :, 0] = bf16((step // 128) * 2.0**-23)[:, :, None]
    bounds[tables[0, :n], :, :, 1] = bf16((step % 128) * 2.0**-30)[:, :, None]
    q = bf16(np.ones((1, hq, d)))
    for blocks in (5, n // 2, n - 1):
        args = (tables, bounds, q, np.array([n * BS]), 0, 1, blocks)
        check(run(gpu_lib, *args), *args)


@pytest.mark.parametrize("n", [40, 100, 700, 3000])
def test_equal_scores_go_to_the_lowest_index(gpu_lib, n):
    rng = np.random.default_rng(n)
    tables, bounds = pool(rng, [n * BS], 2, 64)
    q = rand_bf16(rng, (1, 8, 64))
    same = bounds[tables[0, 0]].copy()
    for dup in (np.arange(n), np.arange(0, n, 2), rng.permutation(n)[:n // 3], np.arange(n - 9, n)):
        b = bounds.copy()
        b[tables[0, dup]] = same
        for blocks in (4, n // 4, n - 2):
            args = (tables, b, q, np.array([n * BS]), 1, 1, blocks)
            check(run(gpu_lib, *args), *args)
    args = (tables, bounds, np.zeros_like(q), np.array([n * BS]), 1, 2, 10)  # all scores zero
    check(run(gpu_lib, *args), *args)
    coarse = bf16(rng.integers(-2, 3, bounds.shape))
    args = (tables, coarse, bf16(rng.integers(-1, 2, q.shape)), np.array([n * BS]), 0, 1, n // 3)
    check(run(gpu_lib, *args), *args)


@pytest.mark.parametrize("n", [75, 200, 900])
def test_values_that_are_not_finite(gpu_lib, n):
    rng = np.random.default_rng(6)
    tables, bounds = pool(rng, [n * BS, n * BS], 2, 128)
    q = rand_bf16(rng, (2, 8, 128))
    b = bounds.copy()
    b[tables[0, 50], 0, 0, 3] = 0x7FC0   # NaN
    b[tables[0, 60], 0, 1, 127] = 0xFF80  # -inf
    b[tables[0, 70], 1, 0, 0] = 0x7F80   # +inf
    args = (tables, b, q, np.array([n * BS] * 2), 1, 2, 6)
    check(run(gpu_lib, *args), *args)
    b[tables[0, :n]] = 0x7FC0  # nothing finite: the lowest indices
    check(run(gpu_lib, *args), *args)
    q[1, 5, 9] = 0x7F80
    check(run(gpu_lib, *args), *args)


@pytest.mark.parametrize("n", [40, 300, 700])
@pytest.mark.parametrize("side", [0, 1])
def test_an_infinite_bound_that_no_query_takes(gpu_lib, n, side):
    """Queries of one sign, which read the other side of the box: the block comes first all the same."""
    rng = np.random.default_rng(8)
    tables, bounds = pool(rng, [n * BS], 1, 128)
    q = rand_bf16(rng, (1, 4, 128)) & 0x7FFF
    if side == 0:
        q |= 0x8000
    b = bounds.copy()
    b[tables[0, n // 2], 0, side, 77] = (0x7F80, 0xFF80)[side]
    args = (tables, b, q, np.array([n * BS]), 1, 1, 4)
    got = run(gpu_lib, *args)
    check(got, *args)
    assert n // 2 in got[0, 0].tolist()


@pytest.mark.parametrize("n", [60, 300, 700])
def test_large_and_tiny_values(gpu_lib, n):
    """Sums that pass the 32-bit range both ways, and products below it."""
    rng = np.random.default_rng(7)
    for scale_q, scale_b in ((2.0**100, 2.0**100), (2.0**-100, 2.0**-60), (2.0**-130, 1.0),
                             (1.0, 2.0**-130), (2.0**120, 1.0)):
        tables, bounds = pool(rng, [n * BS], 2, 64, nan=False)
        bounds = bf16(np.rint(bf16_to_f64(bounds) * 8) * scale_b)
        q = bf16(rng.integers(-8, 9, (1, 4, 64)) * scale_q)
        args = (tables, bounds, q, np.array([n * BS]), 1, 1, 50)
        check(run(gpu_lib, *args), *args)


def test_no_rows_and_no_scores(gpu_lib):
    import torch
    rng = np.random.default_rng(9)
    tables, bounds = pool(rng, [500], 2, 64)
    q = rand_bf16(rng, (1, 4, 64))
    args = (tables, bounds, q, np.array([500]), 3, 5, 8)  # the fixed ones are all
    check(run(gpu_lib, *args), *args)
    check(run(gpu_lib, tables, bounds, q, np.array([0]), 0, 1, 8), tables, bounds, q,
          np.array([0]), 0, 1, 8)
    e = torch.empty((0, 4, 64), dtype=torch.bfloat16, device="cuda")
    gpu_lib.pkv_select_blocks(to_dev_bits(bounds), e, i32(tables), i32([]), 500, 0, 1,
                              torch.empty((0, 2, 3), dtype=torch.int32, device="cuda"),
                              row_seq=i32([]))


def test_bad_ids_read_a_stand_in(gpu_lib):
    """Ids outside the pool give a choice, whichever, within the row."""
    rng = np.random.default_rng(10)
    tables, bounds = pool(rng, [900], 2, 64, nan=False)
    tables[0, ::3] = -5
    tables[0, 1] = len(bounds)
    got = run(gpu_lib, tables, bounds, rand_bf16(rng, (1, 4, 64)), np.array([900]), 1, 1, 7)
    assert ((got >= 0) & (got < 57)).all() and (np.diff(got, axis=2) > 0).all()


def test_replays_and_another_stream(gpu_lib):
    import torch
    lib = gpu_lib
    rng = np.random.default_rng(12)
    lens = np.array([3000, 70, 900])
    tables, bounds = pool(rng, list(lens), 4, 64)
    q = rand_bf16(rng, (3, 16, 64))
    side = torch.cuda.Stream()
    args = (tables, bounds, q, lens, 1, 2, 9)
    check(run(lib, *args, stream=side), *args)
    db, dq, dt, dl = to_dev_bits(bounds), to_dev_bits(q), i32(tables), i32(lens)
    sel = torch.zeros((3, 4, 9), dtype=torch.int32, device="cuda")
    ws = lib.alloc_workspace(lib.pkv_select_workspace_bytes(3, 16, 4, 64, 3000, 9))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            lib.pkv_select_blocks(db, dq, dt, dl, 3000, 1, 2, sel, workspace=ws)
    for _ in range(3):
        q = rand_bf16(rng, q.shape)
        dq.copy_(to_dev_bits(q))
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        check(sel.cpu().numpy(), tables, bounds, q, lens, 1, 2, 9)


def test_validation_names_a_bad_row(gpu_lib):
    lib = gpu_lib
    rng = np.random.default_rng(13)
    tables, bounds = pool(rng, [100, 50], 2, 64)
    q = rand_bf16(rng, (3, 4, 64))
    lib.pkv_set_debug_validate(True)
    try:
        good = (tables, bounds, q, np.array([100, 0, 50]), 0, 1, 3)
        run(lib, *good, row_seq=np.array([0, -1, 1]))
        for row_seq, lens, row in (([0, 2, 1], [1, 1, 1], 1), ([0, 1, 1], [1, 1, 81], 2),
                                   ([1, 0, -2], [50, 100, 1], 1), ([1, 0, -2], [50, 80, 1], 2),
                                   ([1, 0, 0], [65, 1, 1], 0)):
            with pytest.raises(lib.PkvError, match=f"first offending row {row}"):
                run(lib, tables, bounds, q, np.array(lens), 0, 1, 3, row_seq=np.array(row_seq),
                    max_len=80)
    finally:
        lib.pkv_set_debug_validate(False)


@pytest.mark.parametrize("hq,hkv,d", [(32, 8, 128), (16, 4, 64), (16, 1, 128), (4, 4, 64)])
def test_many_rows_of_few_sequences(gpu_lib, hq, hkv, d):
    """Rows enough for whole groups, which end inside sequences: 60 rows of them checked."""
    rng = np.random.default_rng(d)
    lens = [2500, 1700, 900, 2100]
    tables, bounds = pool(rng, lens, hkv, d)
    seq = np.repeat(np.arange(4), [1500, 701, 400, 1100])
    seen = np.concatenate([np.arange(n - m + 1, n + 1) for n, m in
                           zip(lens, (1500, 701, 400, 1100))])
    seq[rng.integers(0, len(seq), 40)] = -1
    q = rand_bf16(rng, (len(seq), hq, d))
    got = run(gpu_lib, tables, bounds, q, seen, 1, 2, 9, row_seq=seq)
    rows = np.sort(rng.permutation(len(seq))[:60])
    check(got[rows], tables, bounds, q[rows], seen[rows], 1, 2, 9, seq[rows])
    assert (got[seq < 0] == -7).all() and (got[seq >= 0][:, :, 0] == 0).all()


def test_two_calls_at_once(gpu_lib):
    """Two streams, each with its own workspace."""
    import torch
    lib = gpu_lib
    rng = np.random.default_rng(14)
    sides = []
    for k in range(2):
        lens = np.array([9000, 4000, 20000 + k])
        tables, bounds = pool(rng, list(lens), 8, 128)
        q = rand_bf16(rng, (3, 32, 128))
        sides.append(dict(host=(tables, bounds, q, lens, 1, 2, 40), stream=torch.cuda.Stream(),
                          dev=(to_dev_bits(bounds), to_dev_bits(q), i32(tables), i32(lens)),
                          sel=torch.zeros((3, 8, 40), dtype=torch.int32, device="cuda"),
                          ws=lib.alloc_workspace(lib.pkv_select_workspace_bytes(3, 32, 8, 128, 20001,
                                                                                40))))
    torch.cuda.synchronize()
    for _ in range(20):
        for s in sides:
            lib.pkv_select_blocks(*s["dev"], 20001, 1, 2, s["sel"], workspace=s["ws"],
                                  stream=s["stream"])
    torch.cuda.synchronize()
    for s in sides:
        check(s["sel"].cpu().numpy(), *s["host"])


def close_boxes(rng, n, d):
    """n boxes whose scores with queries of ones are 0, 1, .. (n - 1 times 2^-8), in random order, by
    sums of large terms that cancel: 32-bit sums are off by more than the scores differ."""
    large = rng.integers(128, 256, (d - 2) // 2) * 2.0 ** rng.integers(-9, 14, (d - 2) // 2)
    terms = np.concatenate([large, -large])
    step = rng.permutation(n)
    box = np.empty((n, d))
    for b in range(n):
        box[b, :2] = step[b] // 128 * 2.0**-1, step[b] % 128 * 2.0**-8
        box[b, 2:] = rng.permutation(terms)
    return bf16(box)


@pytest.mark.parametrize("hq,hkv,d", [(4, 2, 64), (4, 1, 128)])
@pytest.mark.parametrize("n,sink,nans,close,blocks", [
    (40, 1, [0], range(1, 39), 20),                     # (one wave, scores of its own)
    (40, 0, [39], range(0, 39), 20),                    # the row's own block
    (300, 1, [0], range(64, 80), 9),                    # (four waves, both tiles the first one's)
    (700, 1, [0], range(1, 16), 9),                     # (scores of a launch before)
    (3000, 0, [2999], range(2992, 2999), 5)])
def test_a_nan_bound_beside_close_scores(gpu_lib, hq, hkv, d, n, sink, nans, close, blocks):
    """A NaN in a block that is chosen anyway: the others are chosen by their exact scores still."""
    rng = np.random.default_rng(n + d)
    tables, bounds = pool(rng, [n * BS], hkv, d, nan=False)
    at = tables[0]
    bounds[at[:n]] = bf16(np.full(d, -2.0**-6))
    for h in range(hkv):
        bounds[at[close.start:close.stop], h] = close_boxes(rng, len(close), d)[:, None]
    q = bf16(np.ones((1, hq, d)))
    args = (tables, bounds, q, np.array([n * BS]), sink, 1, blocks)
    check(run(gpu_lib, *args), *args)
    bounds[at[nans], :, 0, 5] = 0x7FC0
    check(run(gpu_lib, *args), *args)


@pytest.mark.parametrize("hq,hkv,d", [(4, 2, 64), (4, 1, 128)])
def test_a_nan_bound_that_only_later_rows_see(gpu_lib, hq, hkv, d):
    rng = np.random.default_rng(d)
    n = 600
    tables, bounds = pool(rng, [n * BS], hkv, d, nan=False)
    at = tables[0]
    bounds[at[:n]] = bf16(np.full(d, -2.0**-6))
    for h in range(hkv):
        bounds[at[577:585], h] = close_boxes(rng, 8, d)[:, None]
    bounds[at[595], :, 1, 7] = 0x7FC0
    q = bf16(np.ones((3, hq, d)))
    seen = np.array([586 * BS - 3, 586 * BS, n * BS])
    args = (tables, bounds, q, seen, 0, 1, 5, np.zeros(3, np.int64))
    check(run(gpu_lib, *args), *args)
