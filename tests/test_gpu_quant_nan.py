"""GPU tier: a value that reads back as NaN makes NaN of every row that sees it, also where its weight is too small
for a float, and whatever the order in which the row's largest score and that value are met. The LSE, which no value
enters, stays.

Queries are ones and a token's key is one number in every dim, so that its score is D times the number: the token of
the largest score has 6 (a code of either width), the others 0, and their weights are exp(-6 D), 0 in 32 bits."""
import numpy as np
import pytest

from oracle import quant as Q
from tests.gpu_util import bf16_to_f64, i32, say
from tests.paged_fixture import rand_bf16

pytestmark = pytest.mark.gpu

BS = 16


def caches(rng, n, hkv, d, bits, top, nan):
    """A table, and a pool of n tokens whose key of number top is the largest, without and with the values of token
    nan of kv head 1 as NaN."""
    blocks = -(-n // BS)
    table = rng.permutation(blocks + 2)[:blocks].astype(np.int32)
    k = np.zeros((blocks, hkv, BS, d))
    k[top // BS, :, top % BS] = 6.0
    v = bf16_to_f64(rand_bf16(rng, (blocks, hkv, BS, d)))
    out = []
    for hurt in (False, True):
        if hurt:
            v[nan // BS, 1, nan % BS, d // 2] = np.nan
        cache = np.full((blocks + 2, hkv, Q.slab_bytes(d, bits)), 255, np.uint8)
        cache[table] = Q.blocks(k, v, d, bits)
        out.append(cache)
    return table[None], out


def places(cached, new):
    """(largest, NaN): the NaN in the tile of the largest score, behind it, before it, among the new rows, at the end."""
    n = cached + new
    return [(100, 105), (105, 100), (100, 300), (300, 100), (0, cached + new // 2), (cached + 3, cached + 9),
            (1, 0), (0, n - 1), (n - 1, 0)]


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cached,new,split", [(600, 150, False), (2000, 40, True), (0, 33, False)])
def test_prefill(gpu_lib, bits, d, cached, new, split):
    import torch
    lib = gpu_lib
    hq, hkv, n = 8, 2, cached + new
    rng = np.random.default_rng(bits + d + new)
    q = torch.ones((new, hq, d), dtype=torch.bfloat16, device="cuda")
    need = lib.pkv_quant_prefill_workspace_bytes(1, new, hq, hkv, d, bits, new, n)
    if split:  # (more than one part of a row's keys)
        assert need >= 2 * new * hq * (d + 2) * 4
    ws = lib.alloc_workspace(need) if split else None

    def attend(table, cache):
        out = torch.empty_like(q)
        lse = torch.empty((new, hq), device="cuda")
        lib.pkv_quant_prefill_attention(torch.from_numpy(cache).cuda(), q, i32(table), i32([cached]), i32([0, new]), new, n,
                                        1.0, out, lse=lse, workspace=ws)
        return out, lse

    for top, nan in places(cached, new):
        if max(top, nan) >= n:
            continue
        say(f"[quant nan] prefill, bits {bits}, d {d}, {cached} + {new}: largest {top}, NaN {nan}")
        table, (clean, hurt) = caches(rng, n, hkv, d, bits, top, nan)
        out, lse = attend(table, clean)
        assert torch.isfinite(out).all() and torch.isfinite(lse).all()
        got, got_lse = attend(table, hurt)
        first = max(nan - cached, 0)
        assert torch.isnan(got[first:, hq // 2:]).all()
        got[first:, hq // 2:] = out[first:, hq // 2:]
        assert torch.equal(got.view(torch.int16), out.view(torch.int16)) and torch.equal(got_lse, lse)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("g,n", [(4, 150), (8, 3000), (16, 700)])
def test_decode(gpu_lib, bits, g, n):
    import torch
    lib = gpu_lib
    hkv, d = 2, 128
    rng = np.random.default_rng(bits + g)
    q = torch.ones((1, g * hkv, d), dtype=torch.bfloat16, device="cuda")
    for top, nan in [(100, 105), (105, 100), (0, n - 1), (n - 1, 0), (20, 140)]:
        table, (clean, hurt) = caches(rng, n, hkv, d, bits, top, nan)
        outs = []
        for cache in (clean, hurt):
            out, lse = torch.empty_like(q), torch.empty((1, g * hkv), device="cuda")
            lib.pkv_quant_decode_attention(torch.from_numpy(cache).cuda(), q, i32(table), i32([n]), n, 1.0, out, lse=lse)
            outs.append((out, lse))
        (out, lse), (got, got_lse) = outs
        assert torch.isfinite(out).all() and torch.isfinite(lse).all() and torch.equal(got_lse, lse)
        assert torch.isnan(got[:, g:]).all() and torch.equal(got[:, :g].view(torch.int16), out[:, :g].view(torch.int16))
