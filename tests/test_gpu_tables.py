"""GPU tier: block tables and row metadata built on the GPU (pkv_extend_tables) against a loop
over the tokens, and against the host block pool that hands out the same blocks."""
import numpy as np
import pytest

from tests.gpu_util import i32, say

pytestmark = pytest.mark.gpu

BS = 16


def expect(tables, cached, new, free, used, max_rows):
    """The step token by token; (None, bits) when it must be refused."""
    b, width = tables.shape
    bits = 0
    if any(c < 0 or n < 0 or int(c) + int(n) > 2**31 - 1 for c, n in zip(cached, new)):
        bits |= 8
    c64, n64 = cached.astype(np.int64), new.astype(np.int64)
    if any(n > 0 and -(-(c + n) // BS) > width for c, n in zip(c64, n64)):
        bits |= 2
    if not bits & 8:
        need = int((-(-(c64 + n64) // BS) - -(-c64 // BS)).sum())
        if n64.sum() > max_rows:
            bits |= 4
        if used < 0 or used + need > len(free):
            bits |= 1
    if bits:
        return None, bits
    tables, taken = tables.copy(), used
    slots, seqs, pos = [], [], []
    for i in range(b):
        for p in range(c64[i], c64[i] + n64[i]):
            if p % BS == 0:
                tables[i, p // BS] = free[taken]
                taken += 1
            slots.append(int(tables[i, p // BS]) * BS + p % BS)
            seqs.append(i)
            pos.append(p)
    pad = max_rows - len(slots)
    return dict(tables=tables, used=taken, cu=np.concatenate([[0], np.cumsum(n64)]),
                lens=c64 + n64, slots=np.array(slots + [-1] * pad, np.int64),
                seqs=np.array(seqs + [-1] * pad, np.int64),
                pos=np.array(pos + [-1] * pad, np.int64),
                row_lens=np.array([p + 1 for p in pos] + [0] * pad, np.int64)), 0


def call(lib, tables, cached, new, free, used, max_rows, alias=False, rows=True):
    import torch
    b = len(cached)
    junk = lambda n, dt=torch.int32: torch.full((n,), 77, dtype=dt, device="cuda")
    t, c, n, f, u = i32(tables), i32(cached), i32(new), i32(free), i32([used])
    uo, lens = (u, c) if alias else (junk(1), junk(b))
    cu, status = junk(b + 1), junk(1)
    arrays = dict(slot_map=junk(max_rows, torch.int64), row_seq=junk(max_rows),
                  positions=junk(max_rows), row_lens=junk(max_rows)) if rows else {}
    lib.pkv_extend_tables(t, c, n, f, u, uo, cu, lens, status, max_rows, **arrays)
    torch.cuda.synchronize()
    h = lambda x: x.cpu().numpy()
    return dict(tables=h(t), used=int(uo), cu=h(cu), lens=h(lens), status=int(status),
                slots=h(arrays["slot_map"]) if rows else None,
                seqs=h(arrays["row_seq"]) if rows else None,
                pos=h(arrays["positions"]) if rows else None,
                row_lens=h(arrays["row_lens"]) if rows else None)


def check(got, tables, cached, new, free, used, max_rows):
    want, bits = expect(tables, cached, new, free, used, max_rows)
    assert got["status"] == bits
    if want is None:  # refused: nothing taken, everything padding
        b = len(cached)
        want = dict(tables=tables, used=used, cu=np.zeros(b + 1), lens=cached,
                    slots=np.full(max_rows, -1), seqs=np.full(max_rows, -1),
                    pos=np.full(max_rows, -1), row_lens=np.zeros(max_rows))
    for k, v in want.items():
        if got[k] is not None:
            assert np.array_equal(got[k], v), k


def draw(rng, b, ctx, new_hi, width=None, spare=5, pad=3, zeros=0.2):
    cached = rng.integers(0, ctx + 1, b)
    new = rng.integers(0, new_hi + 1, b)
    new[rng.random(b) < zeros] = 0
    blocks = -(-(cached + new) // BS)
    width = width or int(blocks.max(initial=0)) + 2
    tables = rng.integers(0, 1 << 20, (b, width)).astype(np.int32)
    need = int((blocks - -(-cached // BS)).sum())
    used = int(rng.integers(0, 9))
    free = rng.permutation(used + need + spare).astype(np.int32)
    return tables, cached.astype(np.int32), new.astype(np.int32), free, used, int(new.sum()) + pad


@pytest.mark.parametrize("b,ctx,new_hi", [
    (1, 0, 1), (1, 15, 1), (1, 16, 1), (1, 0, 20000), (3, 40, 40), (64, 4096, 1), (255, 100, 7),
    (256, 33, 16), (257, 64, 3), (1023, 50, 2), (1024, 50, 40), (1025, 20, 3), (2500, 40, 9),
    (4097, 30, 2), (5000, 17, 33)])
def test_matches_a_loop_over_the_tokens(gpu_lib, b, ctx, new_hi):
    rng = np.random.default_rng(b + ctx + new_hi)
    for alias, spare, pad in ((False, 5, 3), (True, 0, 0)):
        step = draw(rng, b, ctx, new_hi, spare=spare, pad=pad)
        say(f"[tables] b={b} ctx<={ctx} new<={new_hi} rows={step[-1]} alias={alias}")
        check(call(gpu_lib, *step, alias=alias), *step)
    check(call(gpu_lib, *step, rows=False), *step)


def test_no_sequences_and_no_tokens(gpu_lib):
    e = np.zeros(0, np.int32)
    step = (np.zeros((0, 4), np.int32), e, e, e, 0, 5)
    check(call(gpu_lib, *step), *step)
    step = (np.full((3, 4), 9, np.int32), i3(5, 0, 16), i3(0, 0, 0), e, 0, 0)
    check(call(gpu_lib, *step), *step)


def i3(*x):
    return np.array(x, np.int32)


@pytest.mark.parametrize("rows", [40, 6000])  # (one launch, two launches)
@pytest.mark.parametrize("cached,new,free,used,width,bits", [
    ((16, 3), (1, 13), 1, 0, 4, 0),            # the last block of the list
    ((16, 3), (1, 14), 1, 0, 4, 1),            # one too few
    ((16, 3), (1, 13), 5, 5, 4, 1),            # all used
    ((16, 3), (1, 13), 5, -1, 4, 1),           # a counter below the list
    ((0, 64), (1, 0), 5, 0, 4, 0),             # a full row that does not grow
    ((0, 64), (1, 1), 5, 0, 4, 2),             # a full row that would
    ((30, 0), (-1, 2), 5, 0, 4, 8),
    ((-16, 0), (2, 2), 5, 0, 4, 8),
    ((2**31 - 1, 0), (1, 2), 5, 0, 4, 10),     # a length past 31 bits, and the row's end
    ((2**31 - 1, 0), (0, 2), 5, 0, 4, 0),      # (its row is not touched)
    ((2**31 - 1, 2**31 - 1), (2**31 - 1, 2**31 - 1), 5, 0, 4, 10),
    ((0, 0), (20000, 0), 5, 0, 4, 7),
])
def test_refusals_change_nothing(gpu_lib, cached, new, free, used, width, bits, rows):
    rng = np.random.default_rng(5)
    tables = rng.integers(0, 99, (2, width)).astype(np.int32)
    step = (tables, i3(*cached), i3(*new), np.arange(100, 100 + free, dtype=np.int32), used, rows)
    assert expect(*step)[1] == bits
    for alias in (False, True):
        check(call(gpu_lib, *step, alias=alias), *step)


def test_takes_the_blocks_the_host_pool_would(gpu_lib):
    """The same growth on the host pool and, from one sequence's reservation, on the GPU."""
    lib = gpu_lib
    rng = np.random.default_rng(11)
    order = rng.permutation(400)
    lens = [0, 5, 16, 31, 100]
    news = [17, 11, 1, 1, 40]

    def start():
        pool = lib.BlockPool(400, 16, free_order=order)
        seqs = [pool.create() for _ in lens]
        for s, n in zip(seqs, lens):
            assert pool.reserve(s, n) == lib.PKV_OK
            pool.commit(s, n)
        return pool, seqs

    pool, seqs = start()
    for s, n in zip(seqs, news):
        assert pool.reserve(s, n) == lib.PKV_OK
    want, _ = pool.block_tables(seqs, 10)
    pool, seqs = start()
    lot = pool.create()
    assert pool.reserve(lot, 12 * 16) == lib.PKV_OK
    free = pool.block_tables([lot], 12)[0][0]
    tables, cached = pool.block_tables(seqs, 10)
    got = call(lib, tables, cached, np.array(news, np.int32), free, 0, sum(news))
    assert got["status"] == 0 and np.array_equal(got["tables"], want)


@pytest.mark.parametrize("b,rows", [(40, 64), (300, 5000)])
def test_a_captured_step_replays_as_a_loop(gpu_lib, b, rows):
    """With the outputs aliased to the inputs, every replay is the next step."""
    import torch
    lib = gpu_lib
    rng = np.random.default_rng(b)
    cached = rng.integers(0, 40, b).astype(np.int32)
    tables = rng.integers(0, 99, (b, 20)).astype(np.int32)
    new = rng.integers(0, 3, b).astype(np.int32)
    free = rng.permutation(200).astype(np.int32)
    t, c, n, f, u = i32(tables), i32(cached), i32(new), i32(free), i32([0])
    cu, status = i32(np.zeros(b + 1)), i32([0])
    slots = torch.zeros(rows, dtype=torch.int64, device="cuda")
    seqs = i32(np.zeros(rows))
    args = (t, c, n, f, u, u, cu, c, status, rows)
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            lib.pkv_extend_tables(*args, slot_map=slots, row_seq=seqs)
    used = 0
    for step in range(4):
        if step == 2:  # other work between the replays
            torch.zeros(1 << 20, device="cuda").sum().item()
        graph.replay()
        torch.cuda.synchronize()
        want, bits = expect(tables, cached, new, free, used, rows)
        assert bits == 0 and int(status) == 0
        tables, used, cached = want["tables"], want["used"], want["lens"].astype(np.int32)
        assert np.array_equal(t.cpu().numpy(), tables) and int(u) == used
        assert np.array_equal(c.cpu().numpy(), cached)
        assert np.array_equal(slots.cpu().numpy(), want["slots"])
        assert np.array_equal(seqs.cpu().numpy(), want["seqs"])
