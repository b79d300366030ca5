"""GPU tier: rotary positions with the append (pkv_rope_append) against the rotation in 64 bits
and an element-by-element placement in the pool.

Tolerance of a turned value y = scale (a cos - b sin): its rounding to bf16 is at most half a
step, 2^-8 |y|. Before it, the angle in turns is exact to 2^-25 (half a turn's rounding to 32 bits)
times 2 pi = 2^-22.3 rad, sine and cosine are off by 2 units of 2^-24, the scale, the two products
and the sum round by 2^-24 each: below 2^-21 (|a| + |b|) |scale| in all. The frequency in turns
and its product with the position each round by 2^-53, relative: 2^-52 |phi| rad more. Values and every other
byte of the pool are compared bit for bit."""
import math

import numpy as np
import pytest

from tests.gpu_util import bf16_to_f64, i32, say, to_dev_bits, to_host_bits
from tests.paged_fixture import rand_bf16

pytestmark = pytest.mark.gpu

BS = 16


def turn(x, pos, axis_of, inv_freq, interleaved, scale):
    """x [rows][heads][d] in 64 bits; returns the turned rows and their error's scale."""
    y, err = x.copy(), np.zeros_like(x)
    half = len(inv_freq)
    for j in range(half):
        a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + half)
        # (long double: the product of a position and a frequency, to well below 2^-24 rad)
        phi = np.longdouble(pos[axis_of[j]]) * np.longdouble(inv_freq[j])
        far = abs(phi).astype(np.float64)[:, None] * 2.0**-52
        phi = np.fmod(phi, 2 * np.arctan2(np.longdouble(0), np.longdouble(-1)))
        phi = phi.astype(np.float64)[:, None]
        y[..., a] = scale * (x[..., a] * np.cos(phi) - x[..., b] * np.sin(phi))
        y[..., b] = scale * (x[..., b] * np.cos(phi) + x[..., a] * np.sin(phi))
        err[..., a] = err[..., b] = (2.0**-21 + far) * (abs(x[..., a]) + abs(x[..., b])) * abs(scale)
    return y, err


def close(got_bits, want, err, what):
    got = bf16_to_f64(got_bits)
    bound = 2.0**-8 * abs(want) + err * (1 + 2.0**-8)
    over = abs(got - want) > bound
    assert not over.any(), (what, int(over.sum()), np.argwhere(over)[:3], got[over][:3],
                            want[over][:3])


def slots_of(rng, seqs, num_blocks, order="rows"):
    """Slots of ragged sequences (cached, new) in blocks in random order; -1 rows between them."""
    perm = rng.permutation(num_blocks)
    slots, pos, used = [], [], 0
    for cached, new in seqs:
        blocks = -(-(cached + new) // BS)
        mine = perm[used:used + blocks]
        used += blocks
        for p in range(cached, cached + new):
            slots.append(int(mine[p // BS]) * BS + p % BS)
            pos.append(p)
    if order == "reversed":
        slots, pos = slots[::-1], pos[::-1]
    if order == "padded":  # a padding row after every fifth, and outside the pool
        out = [(s, p) for s, p in zip(slots, pos)]
        for k in range(len(out) // 5 * 5, -1, -5):
            out.insert(k, (-1 if k % 2 else num_blocks * BS + k, 3))
        slots, pos = zip(*out)
    return np.array(slots, np.int64), np.array(pos, np.int64)


def run(lib, case, seed=0, inplace=False, fused=True, stream=None):
    import torch
    hq, hkv, d = case["heads"]
    rng = np.random.default_rng(seed)
    seqs = case["seqs"]
    nb = sum(-(-(c + n) // BS) for c, n in seqs) + 3
    slots, pos0 = slots_of(rng, seqs, nb, case.get("order", "rows"))
    t = len(slots)
    axes = case.get("axes", 1)
    pos = np.stack([pos0] + [rng.integers(0, 2000, t) for _ in range(axes - 1)])
    if case.get("far"):
        pos = rng.integers(-2**31, 2**31, (axes, t))
        pos[:, :2] = [[2**31 - 1, -2**31]] * axes
    half = case.get("rot", d) // 2
    inv_freq = [1e4 ** (-j / max(half, 1)) for j in range(half)]
    axis_of = [int(a) for a in rng.integers(0, axes, half)] if axes > 1 else [0] * half
    scale = case.get("scale", 1.0)
    rope = lib.rope_spec(inv_freq, axis_of=axis_of, interleaved=case.get("interleaved", False),
                         scale=scale, num_axes=axes)
    q, k, v = (rand_bf16(rng, (t, h, d)) for h in (hq, hkv, hkv))
    pk, pv = rand_bf16(rng, (nb, hkv, d // 8, BS, 8)), rand_bf16(rng, (nb, hkv, d, BS))
    dk, dv = to_dev_bits(pk), to_dev_bits(pv)
    if fused:  # one projection's rows, with 8 elements behind each
        qkv = torch.zeros((t, (hq + 2 * hkv) * d + 8), dtype=torch.bfloat16, device="cuda")
        parts = [qkv[:, a * d:(a + h) * d].unflatten(1, (h, d))
                 for a, h in ((0, hq), (hq, hkv), (hq + hkv, hkv))]
        for dst, src in zip(parts, (q, k, v)):
            dst.copy_(to_dev_bits(src))
    else:
        parts = [to_dev_bits(x) for x in (q, k, v)]
    fill = rand_bf16(rng, (t, hq, d))
    out = parts[0] if inplace else to_dev_bits(fill)
    before = q if inplace else fill
    lib.pkv_rope_append(dk, dv, *parts, torch.from_numpy(slots).cuda(),
                        i32(pos if axes > 1 else pos[0]), rope, out, stream=stream)
    torch.cuda.synchronize()
    live = (slots >= 0) & (slots < nb * BS)
    got_q, got_k, got_v = to_host_bits(out), to_host_bits(dk), to_host_bits(dv)
    args = (pos, axis_of, inv_freq, case.get("interleaved", False), scale)
    want_q, err_q = turn(bf16_to_f64(q), *args)
    want_k, err_k = turn(bf16_to_f64(k), *args)
    assert np.array_equal(got_q[~live], before[~live]), "padding rows"
    close(got_q[live], want_q[live], err_q[live], "q")
    rows_k = got_k[slots[live] // BS, :, :, slots[live] % BS].reshape(-1, hkv, d)
    close(rows_k, want_k[live], err_k[live], "k")
    rot = 2 * half
    assert np.array_equal(got_q[live][..., rot:], q[live][..., rot:])
    assert np.array_equal(rows_k[..., rot:], k[live][..., rot:])
    pv[slots[live] // BS, :, :, slots[live] % BS] = v[live]
    assert np.array_equal(got_v, pv), "v pool"
    got_k[slots[live] // BS, :, :, slots[live] % BS] = 0
    pk[slots[live] // BS, :, :, slots[live] % BS] = 0
    assert np.array_equal(got_k, pk), "the pool's other keys"
    return got_q[live]


RAGGED = [(0, 1), (5, 30), (16, 16), (31, 1), (7, 8), (8, 8), (9, 23), (100, 77), (3, 4)]
CASES = [
    dict(heads=(4, 2, 64), seqs=[(0, 1)]),
    dict(heads=(4, 2, 64), seqs=[(15, 1)]),
    dict(heads=(32, 8, 128), seqs=[(i, 1) for i in range(40)]),
    dict(heads=(32, 8, 128), seqs=RAGGED),
    dict(heads=(8, 8, 64), seqs=RAGGED, interleaved=True),
    dict(heads=(28, 4, 128), seqs=RAGGED, rot=64, interleaved=True, scale=1.25),
    dict(heads=(16, 1, 128), seqs=RAGGED, rot=32, axes=2),
    dict(heads=(5, 5, 64), seqs=RAGGED, rot=0),
    dict(heads=(6, 3, 128), seqs=[(0, 333)], rot=16, axes=3),
    dict(heads=(16, 4, 64), seqs=[(3, 200), (0, 64)], axes=4, interleaved=True),
    dict(heads=(9, 9, 128), seqs=[(11, 50)], scale=-0.5, rot=96),
    dict(heads=(32, 8, 128), seqs=RAGGED, order="reversed"),
    dict(heads=(4, 2, 64), seqs=RAGGED, order="padded", axes=3),
    dict(heads=(40, 20, 128), seqs=RAGGED, order="padded"),
    dict(heads=(32, 8, 128), seqs=[(5, 500), (0, 333), (11, 64)]),  # (windows of 16 rows)
    dict(heads=(8, 8, 64), seqs=[(5, 500), (0, 333), (11, 64)], order="padded", interleaved=True),
    dict(heads=(17, 17, 64), seqs=[(5, 300), (0, 133)], order="reversed", rot=32),
    dict(heads=(4, 2, 64), seqs=[(0, 40)], far=True),
    dict(heads=(4, 2, 128), seqs=[(0, 40)], far=True, axes=3, interleaved=True),
]


@pytest.mark.parametrize("k", range(len(CASES)))
def test_matches_the_rotation_in_64_bits(gpu_lib, k):
    say(f"[rope] {CASES[k]}")
    a = run(gpu_lib, CASES[k])
    b = run(gpu_lib, CASES[k], inplace=True)
    c = run(gpu_lib, CASES[k], fused=False)
    assert np.array_equal(a, b) and np.array_equal(b, c)


def test_another_stream(gpu_lib):
    import torch
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    run(gpu_lib, CASES[3], seed=4, stream=side)


def test_no_rows(gpu_lib):
    import torch
    e = torch.empty((0, 4, 64), dtype=torch.bfloat16, device="cuda")
    kv = torch.zeros((2, 2, 8, BS, 8), dtype=torch.bfloat16, device="cuda")
    vv = torch.zeros((2, 2, 64, BS), dtype=torch.bfloat16, device="cuda")
    gpu_lib.pkv_rope_append(kv, vv, e, e[:, :2], e[:, :2],
                            torch.empty(0, dtype=torch.int64, device="cuda"), i32([]),
                            gpu_lib.rope_spec([1.0] * 32), e)


def test_infinite_and_nan_values_pass(gpu_lib):
    """Values are copied as bits; a NaN or infinity among turned dims stays in its pair."""
    import torch
    d = 64
    q = torch.zeros((1, 1, d), dtype=torch.bfloat16, device="cuda")
    q[0, 0, 3] = math.inf
    q[0, 0, 5] = math.nan
    v = torch.full((1, 1, d), math.nan, dtype=torch.bfloat16, device="cuda")
    kc = torch.zeros((1, 1, d // 8, BS, 8), dtype=torch.bfloat16, device="cuda")
    vc = torch.zeros((1, 1, d, BS), dtype=torch.bfloat16, device="cuda")
    out = torch.empty_like(q)
    gpu_lib.pkv_rope_append(kc, vc, q, q, v, torch.zeros(1, dtype=torch.int64, device="cuda"),
                            i32([1]), gpu_lib.rope_spec([0.1] * 32), out)
    bad = torch.nonzero(~torch.isfinite(out[0, 0])).flatten().tolist()
    assert bad == [3, 5, 35, 37]
    assert torch.isnan(vc[0, 0, :, 0]).all() and (vc[0, 0, :, 1:] == 0).all()


def test_a_captured_append_replays(gpu_lib):
    import torch
    lib = gpu_lib
    rng = np.random.default_rng(3)
    hq, hkv, d, t = 8, 2, 128, 20
    seqs = [(4, 9), (30, 11)]
    slots, pos = slots_of(rng, seqs, 8)
    x = to_dev_bits(rand_bf16(rng, (t, hq + 2 * hkv, d)))
    q, k, v = x.split([hq, hkv, hkv], dim=1)
    kc, vc = (to_dev_bits(rand_bf16(rng, s)) for s in ((8, hkv, d // 8, BS, 8), (8, hkv, d, BS)))
    s, p = torch.from_numpy(slots).cuda(), i32(pos)
    out = torch.empty((t, hq, d), dtype=torch.bfloat16, device="cuda")
    rope = lib.rope_spec([0.5 ** j for j in range(64)])
    args = (q, k, v, s, p, rope)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            lib.pkv_rope_append(kc, vc, *args, out)
    for step in range(3):
        x.copy_(to_dev_bits(rand_bf16(rng, (t, hq + 2 * hkv, d))))
        p.add_(100 * step)
        ek, ev, eo = kc.clone(), vc.clone(), torch.empty_like(out)
        lib.pkv_rope_append(ek, ev, *args, eo)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in ((kc, ek), (vc, ev), (out, eo)):
            assert torch.equal(a.view(torch.int16), b.view(torch.int16))


def test_validation_names_a_bad_slot(gpu_lib):
    import torch
    lib = gpu_lib
    x = torch.zeros((3, 2, 64), dtype=torch.bfloat16, device="cuda")
    kc = torch.zeros((2, 2, 8, BS, 8), dtype=torch.bfloat16, device="cuda")
    vc = torch.zeros((2, 2, 64, BS), dtype=torch.bfloat16, device="cuda")
    args = (i32([0, 1, 2]), lib.rope_spec([1.0] * 32), torch.empty_like(x))
    lib.pkv_set_debug_validate(True)
    try:
        lib.pkv_rope_append(kc, vc, x, x, x, torch.tensor([0, -1, 31]).cuda(), *args)
        with pytest.raises(lib.PkvError, match="slot outside the pool; first offending row 2"):
            lib.pkv_rope_append(kc, vc, x, x, x, torch.tensor([0, -1, 32]).cuda(), *args)
    finally:
        lib.pkv_set_debug_validate(False)
