"""The cache held in 8 or 4 bits, in 64 bits and code by code (include/pkv.h has the format): what a pool's
bytes are for given keys and values, and what they stand for.

A slab's codes are numbered in memory order; key_index and value_index give the number of (dim, slot)."""
import numpy as np

BS = 16
MOST = {8: 448.0, 4: 6.0}
TOP = {8: 119, 4: 125}
TOP_VALUE = {8: 1.125 * 2.0**119, 4: 1.25 * 2.0**125}


def sizes(d, bits):
    """Bytes of key codes, key scales, value codes, value scales."""
    return 2 * d * bits, d // 2, 2 * d * bits, 4 * BS


def slab_bytes(d, bits):
    return sum(sizes(d, bits))


def code_values(bits):
    """What each code stands for."""
    if bits == 4:
        m = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
        return np.concatenate([m, -m])
    c = np.arange(128)
    m = np.where(c < 8, c * 2.0**-9, (8 + c % 8) * 2.0 ** (c // 8 - 10.0))
    m[127] = np.nan
    return np.concatenate([m, -m])


def nearest(y, bits):
    """The code nearest to y (|y| <= M), of two as near the even one; a zero keeps its sign."""
    half = 8 if bits == 4 else 128
    m = code_values(bits)[:half - (bits == 8)]
    a = np.abs(y)
    up = np.clip(np.searchsorted(m, a), 1, len(m) - 1)
    far_up, far_down = m[up] - a, a - m[up - 1]
    code = np.where((far_up < far_down) | ((far_up == far_down) & (up % 2 == 0)), up, up - 1)
    return (code + half * np.signbit(y)).astype(np.uint8)


def key_codes(x, bits):
    """x [.., d]: codes [.., d] and scale bytes [.., d / 32]."""
    g = np.asarray(x, np.float64).reshape(*x.shape[:-1], -1, 32)
    fine = np.isfinite(g).all(-1)
    top = np.abs(np.where(fine[..., None], g, 0)).max(-1)
    held = fine & (top >= 2.0**-100)
    e = np.full(top.shape, TOP[bits])
    for k in range(TOP[bits], -110, -1):  # the least that is not too small
        e = np.where(held & (top <= MOST[bits] * 2.0**k), k, e)
    y = np.clip(np.where(held[..., None], g, 0) / (2.0 ** e.astype(np.float64))[..., None], -MOST[bits], MOST[bits])
    codes = np.where(held[..., None], nearest(y, bits), 0)
    byte = np.where(held, e + 127, np.where(fine, 127, 255))
    return codes.reshape(x.shape).astype(np.uint8), byte.astype(np.uint8)


def value_codes(x, bits):
    """x [.., d]: codes [.., d] and scales [..] (float32)."""
    x = np.asarray(x, np.float64)
    fine = np.isfinite(x).all(-1)
    top = np.abs(np.where(fine[..., None], x, 0)).max(-1)
    held = fine & (top >= 2.0**-100)
    t = np.where(held, top, 1.0)
    e = np.frexp(t / MOST[bits])[1] - 5
    s = np.full(t.shape, np.inf)
    for shift in (1, 0):  # numbers m 2^(e + shift) of 4 significant bits, m = 8 .. 15, about the quotient
        for m in range(16, 7, -1):
            c = m * 2.0 ** (e + shift).astype(np.float64)
            s = np.where((c * MOST[bits] >= t) & (c < s), c, s)
    s = np.minimum(s, TOP_VALUE[bits])
    y = np.clip(np.where(held[..., None], x, 0) / s[..., None], -MOST[bits], MOST[bits])
    codes = np.where(held[..., None], nearest(y, bits), 0)
    scale = np.where(fine, np.where(held, s, 1.0), np.nan)
    return codes.astype(np.uint8), scale.astype(np.float32)


def key_index(d, bits):
    """[16 slots][d]: the number of a key code."""
    per = 128 // bits
    c, slot = np.arange(d)[None, :], np.arange(BS)[:, None]
    return (c // per * BS + slot) * per + c % per


def value_index(d, bits):
    """[16 slots][d]: the number of a value code."""
    planes = 2 if d * bits == 1024 else 1
    run = d // 16 // planes
    c, slot = np.arange(d)[None, :], np.arange(BS)[:, None]
    a, b = c // 16, c % 16
    return (((a // run * 4 + slot // 4) * 16 + b) * run + a % run) * 4 + slot % 4


def _numbered(raw, bits):
    """Bytes as codes in memory order."""
    if bits == 8:
        return raw
    return np.stack([raw & 15, raw >> 4], -1).reshape(*raw.shape[:-1], -1)


def parts(cache, d, bits):
    """cache uint8 [..][slab] as codes [.., 16, d], scale bytes [.., 16, d / 32], codes, scales [.., 16]."""
    kc, ks, vc, _ = sizes(d, bits)
    lead = cache.shape[:-1]
    k = _numbered(cache[..., :kc], bits)[..., key_index(d, bits)]
    e = cache[..., kc:kc + ks].reshape(*lead, BS, d // 32)
    v = _numbered(cache[..., kc + ks:kc + ks + vc], bits)[..., value_index(d, bits)]
    s = np.ascontiguousarray(cache[..., kc + ks + vc:]).view(np.float32)
    return k, e, v, s


def joined(k, e, v, s, d, bits):
    """The bytes of parts."""
    def memory(codes, index):
        flat = np.empty((*codes.shape[:-2], BS * d), np.uint8)
        flat[..., index] = codes
        return flat if bits == 8 else flat[..., 0::2] | flat[..., 1::2] << 4
    lead = k.shape[:-2]
    return np.concatenate([memory(k, key_index(d, bits)), e.reshape(*lead, -1),
                           memory(v, value_index(d, bits)),
                           np.ascontiguousarray(s, dtype=np.float32).view(np.uint8).reshape(*lead, -1)], -1)


def stands_for(cache, d, bits):
    """Keys and values [.., 16, d] in 64 bits."""
    k, e, v, s = parts(cache, d, bits)
    values = code_values(bits)
    scale = np.where(e == 255, np.nan, 2.0 ** (e.astype(np.float64) - 127))
    return values[k] * np.repeat(scale, 32, -1), values[v] * s.astype(np.float64)[..., None]


def written(cache, places, k, v, d, bits):
    """A copy of cache [blocks][hkv][slab] with tokens in it: places [(block, slot)], k, v [n][hkv][d]."""
    cache = cache.copy()
    kc, kb = key_codes(k, bits)
    vc, vs = value_codes(v, bits)
    for n, (block, slot) in enumerate(places):
        pk, pe, pv, ps = (x.copy() for x in parts(cache[block], d, bits))
        pk[:, slot], pe[:, slot], pv[:, slot], ps[:, slot] = kc[n], kb[n], vc[n], vs[n]
        cache[block] = joined(pk, pe, pv, ps, d, bits)
    return cache


def blocks(k, v, d, bits):
    """Slabs [..][slab] of whole blocks' keys and values [.., 16, d]."""
    kc, kb = key_codes(k, bits)
    vc, vs = value_codes(v, bits)
    return joined(kc, kb, vc, vs, d, bits)
