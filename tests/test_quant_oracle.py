"""CPU tier: the quantised cache's oracle against the format's own words, and the exactness that the format
promises."""
import numpy as np
import pytest

from oracle import quant as Q


def bf16(x):
    u = np.asarray(x, np.float32).view(np.uint32)
    return ((u + 0x7FFF + (u >> 16 & 1)) & 0xFFFF0000).view(np.float32).astype(np.float64)


@pytest.mark.parametrize("bits", [4, 8])
def test_codes(bits):
    v = Q.code_values(bits)
    assert np.nanmax(v) == Q.MOST[bits]
    if bits == 8:
        assert v[0x38] == 1 and v[1] == 2.0**-9 and v[8] == 2.0**-6 and v[0x7E] == 448
        assert np.isnan(v[0x7F]) and np.isnan(v[0xFF]) and v[0xB8] == -1
    fine = v[~np.isnan(v)]
    codes = Q.nearest(fine, bits)
    assert np.array_equal(v[codes], fine) and np.array_equal(np.signbit(v[codes]), np.signbit(fine))
    m = np.unique(np.abs(fine))
    for a, b in zip(m[:-1], m[1:]):  # a border goes to the even code, its neighbours to either side
        mid = (a + b) / 2
        c = Q.nearest(np.array([mid, np.nextafter(mid, 0), np.nextafter(mid, 1e9), -mid]), bits)
        assert c[0] % 2 == 0 and v[c[0]] in (a, b)
        assert v[c[1]] == a and v[c[2]] == b and v[c[3]] == -v[c[0]]


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("d", [64, 128])
def test_layout_holds_every_code_once(d, bits):
    for index in (Q.key_index(d, bits), Q.value_index(d, bits)):
        assert np.array_equal(np.sort(index.ravel()), np.arange(16 * d))
    rng = np.random.default_rng(d + bits)
    cache = rng.integers(0, 256, (3, 2, Q.slab_bytes(d, bits)), dtype=np.uint8)
    assert np.array_equal(Q.joined(*Q.parts(cache, d, bits), d, bits), cache)


@pytest.mark.parametrize("bits", [4, 8])
def test_what_codes_stand_for_is_near_and_exact_in_bf16(bits):
    rng = np.random.default_rng(bits)
    x = bf16(rng.standard_normal((300, 128)) * 2.0 ** rng.integers(-90, 110, (300, 1)))
    k, v = Q.stands_for(Q.blocks(x[:288].reshape(18, 16, 128), x[:288].reshape(18, 16, 128), 128, bits), 128, bits)
    x = x[:288].reshape(k.shape)
    assert np.array_equal(bf16(k), k) and np.array_equal(bf16(v), v)
    # a code is off by half its step at most: 2^-4 (2^-2) of itself, or half the least step below the least
    # normal one; a scale is up to 2 (keys) or 1.125 (values) times what the largest value needs
    half, least = (2.0**-4, 2.0**-10) if bits == 8 else (2.0**-2, 0.25)
    top_k = np.abs(x.reshape(18, 16, 4, 32)).max(-1, keepdims=True).repeat(32, -1).reshape(x.shape)
    top_v = np.abs(x).max(-1, keepdims=True)
    assert (np.abs(k - x) <= np.maximum(half * np.abs(x), 2 * least * top_k / Q.MOST[bits])).all()
    assert (np.abs(v - x) <= np.maximum(half * np.abs(x), 1.125 * least * top_v / Q.MOST[bits])).all()


@pytest.mark.parametrize("bits", [4, 8])
def test_edges_of_the_scales(bits):
    most, top = Q.MOST[bits], Q.TOP[bits]
    x = np.zeros((7, 32))
    x[0, 0] = most                   # e = 0 exactly
    x[1, 0] = most * (1 + 2.0**-7)   # one more
    x[2, 0] = 2.0**-100
    x[3, 0] = 2.0**-101              # too small
    x[4, 0] = 2.0**128 * (1 - 2.0**-8)
    x[5, 3] = np.inf
    x[6, 3] = np.nan
    codes, byte = Q.key_codes(x, bits)
    assert byte[0] == [127] and byte[1] == [128] and byte[3] == [127] and byte[4] == [top + 127]
    assert byte[5] == [255] and byte[6] == [255] and not codes[[3, 5, 6]].any()
    assert Q.code_values(bits)[codes[4, 0]] == most
    codes, s = Q.value_codes(x, bits)
    assert s[0] == 1 and s[1] == 1.125 and s[3] == 1 and np.isnan(s[5]) and np.isnan(s[6])
    assert not codes[[3, 5, 6]].any()
    s = s.astype(np.float64)
    m, _ = np.frexp(s[[2, 4]])
    assert np.array_equal(m * 16, np.round(m * 16)) and s[2] * most >= 2.0**-100
    assert s[4] * most < 2.0**128 <= s[4] * most * 1.2 and Q.code_values(bits)[codes[4, 0]] == most
