"""GPU tier: attention over chosen blocks (pkv_sparse_attention) against its definition in 64 bits.

Tolerance, per output element, from the roundings on the way. A score is a 32-bit sum of D exact
products: off by delta = (D + 8) 2^-24 scale sum_d |q_d k_d| at most (the sum's, the scale's and the
exponent's roundings), and a weight by 2 delta relative after the normalisation. A weight is rounded
to bf16 before the value product, half a step 2^-8, and so is the output:
    |error| <= (2^-8 + 2 delta + n 2^-24) sum_p w_p |v_p| + 2^-8 |out|,
n 2^-24 for the sums over n keys in 32 bits. The LSE knows no bf16 weights: delta + n 2^-24 and
2^-21 for exp2, log2 and the result's own roundings (relative to 1 + |lse|)."""
import math

import numpy as np
import pytest

from tests.gpu_util import bf16_to_f64, i32, say, to_dev_bits, to_host_bits
from tests.paged_fixture import rand_bf16

pytestmark = pytest.mark.gpu

BS = 16
NAN = 0x7FC0


def pools(rng, lens, hkv, d):
    """Tables in random order over a pool whose other blocks and tail slots hold NaN."""
    counts = [-(-n // BS) for n in lens]
    nb = sum(counts) + 3
    perm = rng.permutation(nb)
    tables = np.full((len(lens), max(counts) + 1), -1, np.int32)
    pk = np.full((nb, hkv, d // 8, BS, 8), NAN, np.uint16)
    pv = np.full((nb, hkv, d, BS), NAN, np.uint16)
    at = 0
    for i, c in enumerate(counts):
        mine = perm[at:at + c]
        at += c
        tables[i, :c] = mine
        pk[mine] = rand_bf16(rng, (c, hkv, d // 8, BS, 8))
        pv[mine] = rand_bf16(rng, (c, hkv, d, BS))
        if lens[i] % BS:
            pk[mine[-1], :, :, lens[i] % BS:] = NAN
            pv[mine[-1], :, :, lens[i] % BS:] = NAN
    return tables, pk, pv


def lists(rng, lens, hkv, blocks, how="ascending"):
    out = np.full((len(lens), hkv, blocks), -1, np.int32)
    for t, n in enumerate(lens):
        b = -(-max(n, 0) // BS)
        for h in range(hkv):
            k = rng.permutation(b)[:blocks]
            if how == "ascending":
                out[t, h, :len(k)] = np.sort(k)
            else:  # any order, with entries that name nothing between
                e = np.concatenate([k, rng.choice([-1, -9, b, b + 1, 2**31 - 1], blocks)])[:blocks]
                out[t, h] = rng.permutation(e)
    return out


def expect(tables, pk, pv, q, row_lens, sel, scale, row_seq=None):
    """Outputs and LSEs in 64 bits, and the elements' tolerances."""
    t, hq, d = q.shape
    hkv = pk.shape[1]
    g = hq // hkv
    q64 = bf16_to_f64(q)
    out, tol = np.zeros((t, hq, d)), np.zeros((t, hq, d))
    lse, ltol = np.full((t, hq), -math.inf), np.zeros((t, hq))
    for r in range(t):
        s = r if row_seq is None else row_seq[r]
        if s < 0:
            continue
        n = -(-max(row_lens[r], 0) // BS)
        for h in range(hkv):
            keys, vals = [], []
            for b in sel[r, h]:
                if not 0 <= b < min(n, tables.shape[1]) or not 0 <= tables[s, b] < len(pk):
                    continue
                m = min(BS, row_lens[r] - b * BS)
                blk = tables[s, b]
                keys.append(bf16_to_f64(pk[blk, h, :, :m]).transpose(1, 0, 2).reshape(m, d))
                vals.append(bf16_to_f64(pv[blk, h, :, :m]).T)
            if not keys:
                continue
            k, v = np.concatenate(keys), np.concatenate(vals)
            for j in range(h * g, (h + 1) * g):
                z = scale * (k @ q64[r, j])
                delta = (d + 8) * 2.0**-24 * scale * (abs(k) @ abs(q64[r, j])).max()
                top = z.max()
                w = np.exp(z - top)
                total = w.sum()
                w /= total
                out[r, j] = w @ v
                lse[r, j] = top + math.log(total)
                tol[r, j] = (2.0**-8 + 2 * delta + len(k) * 2.0**-24) * (w @ abs(v)) + \
                    2.0**-8 * abs(out[r, j])
                ltol[r, j] = delta + len(k) * 2.0**-24 + 2.0**-21 * (1 + abs(lse[r, j]))
    return out, tol, lse, ltol


def run(lib, tables, pk, pv, q, row_lens, sel, scale, row_seq=None, lse=True, stream=None):
    import torch
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
    ls = torch.full(q.shape[:2], 7.0, device="cuda") if lse else None
    lib.pkv_sparse_attention(to_dev_bits(pk), to_dev_bits(pv), to_dev_bits(q), i32(tables),
                             i32(row_lens), i32(sel), scale, out,
                             row_seq=None if row_seq is None else i32(row_seq), lse=ls,
                             stream=stream)
    torch.cuda.synchronize()
    return to_host_bits(out), ls.cpu().numpy() if lse else None


def check(got, tables, pk, pv, q, row_lens, sel, scale, row_seq=None):
    out, tol, lse, ltol = expect(tables, pk, pv, q, row_lens, sel, scale, row_seq)
    o = bf16_to_f64(got[0])
    live = np.ones(len(q), bool) if row_seq is None else np.asarray(row_seq) >= 0
    assert (o[~live] == 7).all() and (got[1] is None or (got[1][~live] == 7).all())
    err = abs(o - out)[live]
    say(f"  error up to {err.max(initial=0):.2e}, {(err / np.maximum(tol[live], 1e-30)).max(initial=0):.2f} of the tolerance")
    assert (err <= tol[live]).all()
    if got[1] is not None:
        none = np.isneginf(lse)
        assert (np.isneginf(got[1]) == none)[live].all()
        ok = live[:, None] & ~none
        assert (abs(got[1][ok] - lse[ok]) <= ltol[ok]).all()


HEADS = [(4, 2, 64), (32, 8, 128), (8, 8, 64), (16, 1, 128), (28, 4, 128), (3, 1, 64)]


@pytest.mark.parametrize("hq,hkv,d", HEADS)
@pytest.mark.parametrize("lens,blocks", [
    ([1], 1), ([1, 15, 16, 17, 5], 1), ([400, 129, 31, 2000], 3), ([1000, 33, 777], 8),
    ([3000], 65), ([3000, 16 * 150], 128), ([16 * 200] * 3, 200)])
def test_decode_rows(gpu_lib, hq, hkv, d, lens, blocks):
    say(f"[sparse] {hq}/{hkv} heads of {d}, {lens}, {blocks} blocks")
    rng = np.random.default_rng(d + hq)
    pool = pools(rng, lens, hkv, d)
    q = rand_bf16(rng, (len(lens), hq, d))
    for how in ("ascending", "any"):
        args = (*pool, q, np.array(lens), lists(rng, lens, hkv, blocks, how), d ** -0.5)
        got = run(gpu_lib, *args)
        check(got, *args)
        again = run(gpu_lib, *args, lse=False)
        assert np.array_equal(got[0], again[0]), "another run, without LSEs"


@pytest.mark.parametrize("hq,hkv,d", HEADS)
@pytest.mark.parametrize("blocks", [2, 13])
def test_rows_of_longer_suffixes(gpu_lib, hq, hkv, d, blocks):
    rng = np.random.default_rng(hq)
    lens = [900, 40, 1500]
    pool = pools(rng, lens, hkv, d)
    seq, seen = [], []
    for s, n in ((0, 37), (1, 9), (2, 50)):
        seq += [s] * n
        seen += list(range(lens[s] - n + 1, lens[s] + 1))
    seq[3] = seq[20] = seq[60] = -1
    seen[5], seen[70], seen[6], seen[71] = 0, -3, 1, 200
    q = rand_bf16(rng, (len(seq), hq, d))
    sel = lists(rng, seen, hkv, blocks, "any")
    sel[8] = -1  # nothing listed
    args = (*pool, q, np.array(seen), sel, d ** -0.5, np.array(seq))
    check(run(gpu_lib, *args), *args)


def test_many_rows(gpu_lib):
    """Enough rows that each wave is alone, one of them long."""
    rng = np.random.default_rng(1)
    lens = [700] * 299 + [4000]
    pool = pools(rng, lens, 8, 64)
    q = rand_bf16(rng, (300, 8, 64))
    args = (*pool, q, np.array(lens), lists(rng, lens, 8, 20, "any"), 0.125)
    check(run(gpu_lib, *args), *args)


def test_all_blocks_is_the_decode(gpu_lib):
    """Every block listed: as pkv_decode_attention, each within the tolerance of 64 bits."""
    import torch
    lib = gpu_lib
    rng = np.random.default_rng(2)
    hq, hkv, d = 32, 8, 128
    lens = np.array([1000, 17, 320])
    tables, pk, pv = pools(rng, list(lens), hkv, d)
    q = rand_bf16(rng, (3, hq, d))
    sel = np.full((3, hkv, 63), -1, np.int32)
    for t, n in enumerate(lens):
        sel[t, :, :-(-n // BS)] = np.arange(-(-n // BS))
    args = (tables, pk, pv, q, lens, sel, d ** -0.5)
    check(run(lib, *args), *args)
    out = torch.empty((3, hq, d), dtype=torch.bfloat16, device="cuda")
    lse = torch.empty((3, hq), device="cuda")
    lib.pkv_decode_attention(to_dev_bits(pk), to_dev_bits(pv), to_dev_bits(q), i32(tables),
                             i32(lens), 1000, d ** -0.5, out, lse=lse)
    check((to_host_bits(out), lse.cpu().numpy()), *args)


def test_special_values(gpu_lib):
    """Scores of -infinity weigh nothing, all of them give zeros; a NaN among the visible keys
    or values reaches its heads' outputs and no others'."""
    rng = np.random.default_rng(3)
    hq, hkv, d = 4, 2, 64
    lens = [40, 40, 40, 40]
    tables, pk, pv = pools(rng, lens, hkv, d)
    q = rand_bf16(rng, (4, hq, d))
    q[:, :, 0] = 0x3F80  # 1
    pk[tables[0, 0], :, 0, 3, 0] = 0xFF80  # one key of -inf
    for b in range(3):
        pk[tables[1, b], :, 0, :, 0] = 0xFF80  # every key
    pv[tables[1, 0], 0, 5, 2] = 0x7F80  # (an infinite value of no weight)
    pk[tables[2, 1], 0, 0, 3, 0] = NAN
    pv[tables[3, 2], 1, 9, 1] = NAN
    sel = np.tile(np.arange(3, dtype=np.int32), (4, hkv, 1))
    got, lse = run(gpu_lib, tables, pk, pv, q, np.array(lens), sel, 0.125)
    o = bf16_to_f64(got)
    assert np.isfinite(o[0]).all() and (o[1] == 0).all() and np.isneginf(lse[1]).all()
    assert np.isnan(o[2, :2]).all() and np.isfinite(o[2, 2:]).all()
    assert np.isnan(o[3, 2:, 9]).all() and np.isfinite(np.delete(o[3], 9, axis=1)).all()
    # the same key hidden, by the list and by the row's length
    sel[2, :, 1] = -1
    got, _ = run(gpu_lib, tables, pk, pv, q, np.array([40, 40, 40, 33]), sel, 0.125)
    assert np.isfinite(bf16_to_f64(got)).all()


def test_table_entries_outside_the_pool_are_passed_over(gpu_lib):
    rng = np.random.default_rng(4)
    tables, pk, pv = pools(rng, [500], 2, 128)
    tables[0, 3], tables[0, 7] = -1, len(pk)
    q = rand_bf16(rng, (1, 8, 128))
    args = (tables, pk, pv, q, np.array([500]), lists(rng, [500], 2, 32), 0.1)
    check(run(gpu_lib, *args), *args)


def test_a_row_length_past_the_table(gpu_lib):
    """Lengths far past the table's row see the table's blocks, each of them whole."""
    rng = np.random.default_rng(5)
    tables, pk, pv = pools(rng, [16 * 5], 2, 64)
    tables = tables[:, :5].copy()
    q = rand_bf16(rng, (1, 4, 64))
    for n in (81, 2**31 - 1):
        args = (tables, pk, pv, q, np.array([n]), np.arange(7, dtype=np.int32).reshape(1, 1, 7)
                .repeat(2, 1), 0.125)
        check(run(gpu_lib, *args), *args)


def test_a_pool_past_4_gb(gpu_lib):
    import torch
    lib = gpu_lib
    rng = np.random.default_rng(6)
    hkv, d, nb = 8, 128, 150000  # 4.9 GB of keys
    n = 700
    tables, pk, pv = pools(rng, [n], hkv, d)
    ids = np.concatenate([nb - 1 - np.arange(30), np.arange(len(pk) - 30)]).astype(np.int64)
    dk = torch.zeros((nb, hkv, d // 8, BS, 8), dtype=torch.bfloat16, device="cuda")
    dv = torch.zeros((nb, hkv, d, BS), dtype=torch.bfloat16, device="cuda")
    dk[torch.from_numpy(ids).cuda()] = to_dev_bits(pk)
    dv[torch.from_numpy(ids).cuda()] = to_dev_bits(pv)
    far = np.where(tables >= 0, ids[tables], -1).astype(np.int32)
    q = rand_bf16(rng, (1, 32, d))
    sel = lists(rng, [n], hkv, 40)
    out = torch.empty((1, 32, d), dtype=torch.bfloat16, device="cuda")
    lib.pkv_sparse_attention(dk, dv, to_dev_bits(q), i32(far), i32([n]), i32(sel), 0.09, out)
    near = run(lib, tables, pk, pv, q, np.array([n]), sel, 0.09)
    assert np.array_equal(to_host_bits(out), near[0]), "placement changes nothing"
    check(near, tables, pk, pv, q, np.array([n]), sel, 0.09)


def test_replays_and_another_stream(gpu_lib):
    import torch
    lib = gpu_lib
    rng = np.random.default_rng(7)
    lens = np.array([3000, 70, 900])
    tables, pk, pv = pools(rng, list(lens), 4, 64)
    sel = lists(rng, list(lens), 4, 100)
    q = rand_bf16(rng, (3, 16, 64))
    side = torch.cuda.Stream()
    args = (tables, pk, pv, q, lens, sel, 0.125)
    check(run(lib, *args, stream=side), *args)
    dk, dv, dq, dt, dl, ds = (to_dev_bits(pk), to_dev_bits(pv), to_dev_bits(q), i32(tables),
                              i32(lens), i32(sel))
    out = torch.zeros((3, 16, 64), dtype=torch.bfloat16, device="cuda")
    ws = lib.alloc_workspace(lib.pkv_sparse_workspace_bytes(3, 16, 4, 64, 100))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            lib.pkv_sparse_attention(dk, dv, dq, dt, dl, ds, 0.125, out, workspace=ws)
    for _ in range(3):
        q = rand_bf16(rng, q.shape)
        dq.copy_(to_dev_bits(q))
        if ws is not None:
            ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        eager = run(lib, tables, pk, pv, q, lens, sel, 0.125)
        assert np.array_equal(to_host_bits(out), eager[0])
        check(eager, tables, pk, pv, q, lens, sel, 0.125)


def test_no_rows(gpu_lib):
    import torch
    rng = np.random.default_rng(8)
    tables, pk, pv = pools(rng, [50], 2, 64)
    e = torch.empty((0, 4, 64), dtype=torch.bfloat16, device="cuda")
    gpu_lib.pkv_sparse_attention(to_dev_bits(pk), to_dev_bits(pv), e, i32(tables), i32([]),
                                 torch.empty((0, 2, 3), dtype=torch.int32, device="cuda"), 0.1, e,
                                 row_seq=i32([]))


def kinds(x):
    """0 where finite, 1 and -1 for the infinities, 2 for NaN."""
    return np.where(np.isnan(x), 2, np.where(np.isinf(x), np.sign(x), 0))


@pytest.mark.parametrize("hq,hkv,d", [(2, 2, 64), (8, 2, 128), (16, 2, 64), (16, 1, 128), (28, 4, 128)])
@pytest.mark.parametrize("lens,blocks", [([40, 170], 12), ([3000, 16 * 150], 188), ([60] * 300, 4)])
def test_infinite_values_of_positive_weight(gpu_lib, hq, hkv, d, lens, blocks):
    """An infinite value at a visible key makes its dim infinite (NaN where both infinities meet) for
    every head of its kv head, however many these are, as in pkv_decode_attention; the other dims
    stay within their tolerance, and a value that the list or the length hides changes nothing. A wave
    of its own per row, four waves, and splits."""
    import torch
    lib = gpu_lib
    rng = np.random.default_rng(d + hq)
    tables, pk, pv = pools(rng, lens, hkv, d)
    q = rand_bf16(rng, (len(lens), hq, d))
    lens = np.array(lens)
    n = -(-lens // BS)
    for t in range(len(lens)):
        for dim, bits, block in ((3, 0x7F80, 0), (17, 0xFF80, 1), (40, 0x7F80, n[t] - 1),
                                 (50, 0x7F80, 0), (50, 0xFF80, 2)):
            slot = rng.integers(0, (lens[t] - 1) % BS + 1)
            pv[tables[t, block], hkv - 1, dim, slot] = bits
    sel = np.full((len(lens), hkv, blocks), -1, np.int32)
    for t in range(len(lens)):
        sel[t, :, :n[t]] = np.arange(n[t])
    args = (tables, pk, pv, q, lens, sel, d ** -0.5)
    out, lse = run(lib, *args)
    with np.errstate(invalid="ignore"):
        want, tol, want_lse, ltol = expect(*args)
    got = bf16_to_f64(out)
    assert np.array_equal(kinds(got), kinds(want))
    fine = np.isfinite(want)
    assert (abs(got[fine] - want[fine]) <= tol[fine]).all() and (abs(lse - want_lse) <= ltol).all()
    g = hq // hkv
    for dim, kind in ((3, 1), (17, -1), (40, 1), (50, 2)):
        assert (kinds(got[:, -g:, dim]) == kind).all()
    assert np.isfinite(got[:, :hq - g]).all()
    dense = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")
    lib.pkv_decode_attention(to_dev_bits(pk), to_dev_bits(pv), to_dev_bits(q), i32(tables), i32(lens),
                             int(lens.max()), d ** -0.5, dense)
    assert np.array_equal(kinds(bf16_to_f64(to_host_bits(dense))), kinds(got))
    # hidden by the list, and by the row's length
    sel[:, :, :3] = -1
    hide = np.maximum(n - 1, 0) * BS
    got = run(lib, tables, pk, pv, q, hide, sel, d ** -0.5)[0]
    assert np.isfinite(bf16_to_f64(got)).all()


@pytest.mark.parametrize("hq,hkv,d", [(2, 2, 64), (8, 2, 128), (16, 2, 64), (16, 1, 128), (28, 4, 128)])
@pytest.mark.parametrize("lens,blocks", [([90, 33], 6), ([100, 160], 10), ([16 * 100], 100),
                                         ([60] * 300, 4)])
def test_weights_keep_more_than_bf16(gpu_lib, hq, hkv, d, lens, blocks):
    """Weights reach the value product in two bf16 parts, off by 2^-16 of themselves, 2 n products per
    element whose sums are off by 2^-23 an addition, and some 2^-24 for exp2, division and rescaling:
        |error| <= (2^-16 + 2 delta + (5 n + 32) 2^-24) sum_p w_p |v_p| + 2^-8 |out|.
    Weights rounded once (2^-8) are past this where values cancel."""
    rng = np.random.default_rng(d + hq)
    tables, pk, pv = pools(rng, lens, hkv, d)
    q = rand_bf16(rng, (len(lens), hq, d))
    lens = np.array(lens)
    args = (tables, pk, pv, q, lens, lists(rng, lens, hkv, blocks), 2 * d ** -0.5)
    want, loose = expect(*args)[:2]
    n = (-(-lens // BS)).clip(max=blocks)[:, None, None] * BS
    # (the looser tolerance less its share of rounded weights, and the sums' share)
    weight = np.zeros_like(want)
    for r in range(len(lens)):  # sum_p w_p |v_p|
        weight[r] = expect(tables, pk, pv & 0x7FFF, q[r:r + 1], lens[r:r + 1], args[5][r:r + 1], args[6],
                           [r])[0][0]
    delta2 = (loose - 2.0**-8 * abs(want)) / weight - 2.0**-8  # (2 delta + n 2^-24, n visible keys)
    tol = (2.0**-16 + delta2 + (4 * n + 32) * 2.0**-24) * weight + 2.0**-8 * abs(want)
    err = abs(bf16_to_f64(run(gpu_lib, *args)[0]) - want)
    say(f"  {(err / tol).max():.2f} of the tolerance")
    assert (err <= tol).all()


@pytest.mark.parametrize("hq,hkv,d", [(4, 4, 64), (8, 2, 128), (16, 2, 64), (16, 1, 128)])
def test_values_near_the_largest(gpu_lib, hq, hkv, d):
    """A value of 2^126 at a score that passes the earlier ones by 7 (base 2): its weight is 1 in the end
    and the sums stay finite, as in pkv_decode_attention, for each sign. (Keys of the earlier steps hold
    ordinary values: 64 of 2^126 with a weight of 1 would pass the 32-bit range in any order.)"""
    import torch
    lib = gpu_lib
    rng = np.random.default_rng(d)
    lens = np.array([75])
    tables, pk, pv = pools(rng, list(lens), hkv, d)
    pk[tables[0, :5]] = 0
    pk[tables[0, 4], :, 0, 6, 0] = 0x3F80  # 1
    pv[tables[0, 4], :, :, 6] = np.where(rng.integers(0, 2, (hkv, d)), 0x7E80, 0xFE80)
    q = np.zeros((1, hq, d), np.uint16)
    q[:, :, 0] = 0x40E0  # 7
    args = (tables, pk, pv, q, lens, np.arange(5, dtype=np.int32).reshape(1, 1, 5).repeat(hkv, 1),
            math.log(2))
    check(run(lib, *args), *args)
    out = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")
    lib.pkv_decode_attention(to_dev_bits(pk), to_dev_bits(pv), to_dev_bits(q), i32(tables), i32(lens), 75,
                             math.log(2), out)
    check((to_host_bits(out), None), *args)


def test_validation_takes_what_the_call_passes_over(gpu_lib):
    """Table entries outside the pool and lengths past the table are in order; rows of no sequence and
    negative lengths are not."""
    lib = gpu_lib
    rng = np.random.default_rng(15)
    tables, pk, pv = pools(rng, [500, 80], 2, 64)
    tables = tables[:, :31].copy()
    tables[0, 3], tables[0, 7] = -1, len(pk)
    q = rand_bf16(rng, (4, 4, 64))
    seen, seq = np.array([500, 2**31 - 1, 0, 64]), np.array([0, 0, -1, 1])
    sel = lists(rng, [496, 496, 496, 64], 2, 32, "any")
    args = (tables, pk, pv, q, seen, sel, 0.1, seq)
    pk[tables[0, 30], :, :, 4:] = 0  # (slots that the second row sees)
    pv[tables[0, 30], :, :, 4:] = 0
    off = run(lib, *args)
    check(off, *args)
    lib.pkv_set_debug_validate(True)
    try:
        on = run(lib, *args)
        assert all(np.array_equal(a, b) for a, b in zip(off, on))
        for bad_seen, bad_seq, row in (([500, -1, 0, 64], [0, 0, -1, 1], 1),
                                       ([500, 9, 0, 64], [0, 0, -2, 1], 2),
                                       ([500, 9, 0, 64], [0, 0, 0, 2], 3)):
            with pytest.raises(lib.PkvError, match=f"first offending row {row}"):
                run(lib, tables, pk, pv, q, np.array(bad_seen), sel, 0.1, np.array(bad_seq))
    finally:
        lib.pkv_set_debug_validate(False)


@pytest.mark.parametrize("hq,hkv,d", [(4, 1, 64), (6, 3, 64), (16, 1, 128)])
@pytest.mark.parametrize("n,blocks", [(16 * 1100, 1040), (16 * 2100 - 7, 1360), (16 * 4096, 2048),
                                      (16 * 4096, 4096), (16 * 1500, 65536)])
def test_long_lists_of_one_row(gpu_lib, hq, hkv, d, n, blocks):
    """Few rows with more than 1024 blocks: as many splits as the merge has lanes."""
    rng = np.random.default_rng(n + d)
    pool = pools(rng, [n], hkv, d)
    q = rand_bf16(rng, (1, hq, d))
    for how in ("ascending", "any"):
        args = (*pool, q, np.array([n]), lists(rng, [n], hkv, blocks, how), d ** -0.5)
        got = run(gpu_lib, *args)
        check(got, *args)
        row_seq = run(gpu_lib, *args, np.array([0]))
        assert all(np.array_equal(a, b) for a, b in zip(got, row_seq)), "with row_seq"


@pytest.mark.parametrize("hq,hkv,d", [(4, 1, 64), (32, 8, 128), (28, 4, 128), (6, 3, 64)])
def test_splits_of_rows_that_share_a_sequence(gpu_lib, hq, hkv, d):
    """Few rows of longer suffixes with long lists: several workgroups an item, in the XCDs' order."""
    rng = np.random.default_rng(hq)
    lens = [3000, 900]
    pool = pools(rng, lens, hkv, d)
    seq = np.array([0, 0, -1, 0, 1])
    seen = np.array([2998, 2999, 50, 3000, 900])
    q = rand_bf16(rng, (5, hq, d))
    args = (*pool, q, seen, lists(rng, seen, hkv, 180, "any"), d ** -0.5, seq)
    assert gpu_lib.pkv_sparse_workspace_bytes(5, hq, hkv, d, 180) > 0
    check(run(gpu_lib, *args), *args)
