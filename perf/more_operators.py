"""Timed cases of the operators of a paged cache held in 8 or 4 bits: new tokens quantised as they are
appended, blocks of the 16-bit pool quantised and read back, and decode and prefill attention over the
quantised cache.

The cache is uint8 [num_blocks][kv heads][slab]. A slab holds a block's 16 tokens for one kv head: key
codes, key scales, value codes, value scales. With codes of e4m3 (8 bits, largest value M = 448) or e2m1
(4 bits, M = 6; the first of two codes in a byte's low half):

  * keys, per token and 32 dims: e is the least integer with max|x| <= M 2^e (at most 119 for 8 bits and
    125 for 4, where codes saturate), a code stands for x 2^-e rounded to nearest even, the scale byte is
    e + 127. Below max|x| = 2^-100 the codes are 0 and the byte 127; where a value is not finite the codes
    are 0 and the byte is 255, which makes all 32 NaN.
  * values, per token: s is the least number of 4 significant bits that is not below max|x| / M (at most
    1.125 2^119 for 8 bits and 1.25 2^125 for 4, where codes saturate), kept as a float, a code stands for
    x / s rounded to nearest even. Below 2^-100: codes 0 and s = 1; not finite: codes 0 and s = NaN.
  * key codes are [dims in units of 16 bytes][16 slots][unit], key scales [16 slots][dims / 32], value
    codes [planes][4 quarters][16][dims / 16 / planes][4 slots of the quarter] where dim 16 a + b of slot
    4 q + j is entry b of quarter q, a, j (two planes with 8 bits and 128 dims, otherwise one), value scales
    16 floats.

Every code is fully determined: no product or quotient that decides one can fall on the other side of a
border by a 32-bit rounding. So the quantised cache is returned as it is held: codes of 8 bits and the
value scales as numbers, codes of 4 bits (for which torch has no type) and the keys' exponents as bytes.

A case is one call of one operator; prepare() draws lengths, block placement and contents from the seed.
With `own` false run() computes the operators in elementary torch operations in 32 bits. With `own` true it
makes the library's calls. exact() goes from the definitions in 64 bits."""
import math

import numpy as np
import torch

own = False

BS = 16  # tokens per block
MOST = {8: 448.0, 4: 6.0}  # the largest value of a code
TOP = {8: 119, 4: 125}     # the largest exponent of a key scale
TOP_VALUE = {8: 1.125 * 2.0 ** 119, 4: 1.25 * 2.0 ** 125}  # the largest value scale


# ----------------------------------------------------------------------------------------
# the cases
# ----------------------------------------------------------------------------------------
def listed():
    return [
        # a decode step's new tokens, one for each sequence of an ordinary batch
        dict(name="append_step", kind="append", bits=8, hkv=8, d=128, seqs=64, ctx_lo=256, ctx_hi=4096,
             new_lo=1, new_hi=1),
        # documents prefilled once and kept narrow
        dict(name="append_documents", kind="append", bits=4, hkv=8, d=128, seqs=32, ctx_lo=0, ctx_hi=511,
             new_lo=1024, new_hi=8192),
        # one tuple's prefix goes from the 16-bit pool into the narrow one
        dict(name="park_prefix", kind="park", bits=4, hkv=8, d=128, blocks=62),
        # the prefixes of a whole stage, kept for its successor
        dict(name="park_stage", kind="park", bits=8, hkv=4, d=64, blocks=40009),
        # one tuple's prefix comes back for an operator that reads the 16-bit pool
        dict(name="restore_prefix", kind="restore", bits=8, hkv=8, d=128, blocks=62),
        # a stage's prefixes come back
        dict(name="restore_stage", kind="restore", bits=4, hkv=8, d=128, blocks=16411),
        # the smallest step: a few short contexts
        dict(name="decode_few", kind="decode", bits=8, hq=16, hkv=4, d=64, seqs=5, ctx_lo=300, ctx_hi=1003,
             lse=False),
        # one interactive request over a very long context
        dict(name="decode_one", kind="decode", bits=4, hq=32, hkv=8, d=128, seqs=1, ctx_lo=120011,
             ctx_hi=120011, lse=False),
        # an ordinary decode batch
        dict(name="decode_batch", kind="decode", bits=8, hq=32, hkv=8, d=128, seqs=256, ctx_lo=512,
             ctx_hi=4096, lse=True),
        # a decode batch over long documents
        dict(name="decode_documents", kind="decode", bits=4, hq=64, hkv=8, d=128, seqs=64, ctx_lo=8192,
             ctx_hi=32768, lse=False),
        # a downstream operator's suffixes over its tuples' prefixes
        dict(name="prefill_suffixes", kind="prefill", bits=4, hq=32, hkv=8, d=128, seqs=48, ctx_lo=500,
             ctx_hi=3500, new_lo=64, new_hi=401, lse=False),
        # a few suffixes behind long documents
        dict(name="prefill_documents", kind="prefill", bits=8, hq=16, hkv=4, d=64, seqs=3, ctx_lo=4096,
             ctx_hi=16384, new_lo=101, new_hi=509, lse=True),
    ]


_HEADS = [(4, 2, 64), (8, 8, 64), (16, 4, 64), (32, 8, 128), (64, 8, 128), (16, 16, 128), (16, 1, 128),
          (28, 4, 128)]


def _log_int(rng, lo, hi):
    """An integer of lo .. hi, evenly over the logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["append", "park", "restore", "decode", "decode", "decode", "prefill", "prefill"])
    most = {k: max(work(c)[k] for c in listed() if c["kind"] == kind) for k in ("bytes", "flops")}
    while True:
        hq, hkv, d = rng.choice(_HEADS)
        c = dict(kind=kind, bits=rng.choice([4, 8]), hkv=hkv, d=d)
        if kind in ("park", "restore"):
            c.update(blocks=_log_int(rng, 1, 40009))
        else:
            hi = _log_int(rng, 16, 131072)
            c.update(seqs=_log_int(rng, 1, 512), ctx_lo=rng.randint(1, hi), ctx_hi=hi)
        if kind == "append":
            new_hi = rng.choice([1, _log_int(rng, 2, 8192)])
            c.update(new_lo=rng.randint(1, new_hi), new_hi=new_hi)
        if kind == "prefill":
            new_hi = _log_int(rng, 1, 2048)
            c.update(new_lo=rng.randint(1, new_hi), new_hi=new_hi)
        if kind in ("decode", "prefill"):
            c.update(hq=hq, lse=rng.random() < 0.3)
        if "seqs" in c and c["seqs"] * (c["ctx_hi"] + c.get("new_hi", 0)) * hkv * d > 2.2e9:
            continue
        w = work(c)
        if w["bytes"] <= most["bytes"] and w["flops"] <= most["flops"]:
            return c


# ----------------------------------------------------------------------------------------
# the slab
# ----------------------------------------------------------------------------------------
def _sizes(d, bits):
    """Bytes of a slab's key codes, key scales, value codes and value scales."""
    return 2 * d * bits, d // 2, 2 * d * bits, 4 * BS


def _parts(cache, d, bits):
    """Views of the cache's four parts."""
    nb, hkv = cache.shape[:2]
    kc, ks, vc, vs = _sizes(d, bits)
    k = cache[..., :kc].view(nb, hkv, kc // 256, BS, 16)
    e = cache[..., kc:kc + ks].view(nb, hkv, BS, d // 32)
    planes = 2 if bits * d == 1024 else 1
    v = cache[..., kc + ks:kc + ks + vc].view(nb, hkv, planes, 4, 16, d // 16 // planes, bits // 2)
    s = cache[..., kc + ks + vc:].view(torch.float32)
    return k, e, v, s


def _shown(cache, d, bits):
    """The cache as outputs."""
    k, e, v, s = _parts(cache, d, bits)
    if bits == 8:
        k, v = k.view(torch.float8_e4m3fn), v.view(torch.float8_e4m3fn)
    return k, e, v, s


def _split(codes, bits):
    """The last dim's bytes as one code each."""
    if bits == 8:
        return codes
    return torch.stack((codes & 15, codes >> 4), dim=-1).flatten(-2)


def _join(codes, bits):
    if bits == 8:
        return codes
    return codes[..., 0::2] | codes[..., 1::2] << 4


def _key_codes(k, bits):
    """[.., units, slots, bytes] as codes [.., slots, dims]."""
    return _split(k, bits).transpose(-3, -2).flatten(-2)


def _key_bytes(codes, d, bits):
    return _join(codes, bits).unflatten(-1, (2 * d * bits // 256, 16)).transpose(-3, -2)


def _value_codes(v, bits):
    """[.., planes, quarters, 16, dims / 16 / planes, bytes] as codes [.., slots, dims]."""
    n = v.dim() - 5
    x = _split(v, bits)                             # [.., planes, quarters, b, a, j]
    x = x.permute(*range(n), n + 1, n + 4, n, n + 3, n + 2)
    return x.flatten(n, n + 1).flatten(n + 1)


def _value_bytes(codes, d, bits):
    n = codes.dim() - 2
    planes = 2 if bits * d == 1024 else 1
    x = codes.unflatten(-1, (planes, d // 16 // planes, 16)).unflatten(-4, (4, 4))
    x = x.permute(*range(n), n + 2, n, n + 4, n + 3, n + 1)
    return _join(x, bits)


def _values(codes, bits):
    """What codes stand for, in 32 bits."""
    if bits == 8:
        return codes.view(torch.float8_e4m3fn).float()
    mag = (codes & 7).float()
    mag = torch.where(mag < 4, mag / 2, torch.where(mag < 6, mag - 2, 2 * mag - 8))
    return torch.where(codes >= 8, -mag, mag)


# ----------------------------------------------------------------------------------------
# lengths, tables and contents
# ----------------------------------------------------------------------------------------
def _strata(rng, n, lo, hi):
    """n lengths of lo .. hi, one per stratum, shuffled."""
    u = (np.arange(n) + 0.5) / n
    rng.shuffle(u)
    return np.minimum(lo + np.floor(u * (hi - lo + 1)), hi).astype(np.int64)


def _i32(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()


def _tables(rng, lens):
    """Block tables of sequences of these lengths and the pool's size: the blocks in random order, an
    eighth of the pool or more no sequence's."""
    counts = -(-lens // BS)
    total = int(counts.sum())
    most = int(lens.sum()) // BS + len(lens)
    num_blocks = most + most // 8 + 1
    order = rng.permutation(num_blocks)[:total].astype(np.int32)
    tables = np.full((len(lens), int(counts.max())), -1, np.int32)
    at = 0
    for i, n in enumerate(counts):
        tables[i, :n] = order[at:at + n]
        at += n
    return tables, num_blocks


def _randn(gen, *shape):
    """N(0, 1) in bf16, the large ones piece by piece."""
    out = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
    flat = out.view(-1)
    step = 1 << 28
    for a in range(0, flat.numel(), step):
        n = min(step, flat.numel() - a)
        flat[a:a + n] = torch.randn(n, generator=gen, device="cuda")
    return out


def _keys(gen, rows, hkv, d):
    """Keys about a mean per channel, some channels much wider than the others, as cached keys have them."""
    x = _randn(gen, rows, hkv, d)
    wide = torch.exp(0.5 * torch.randn((1, hkv, d), generator=gen, device="cuda"))
    mean = torch.randn((1, hkv, d), generator=gen, device="cuda")
    step = max(1, (1 << 27) // (hkv * d))
    for a in range(0, rows, step):
        x[a:a + step] = x[a:a + step] * wide + mean
    return x


def _cache(gen, num_blocks, hkv, d, bits):
    """A quantised pool whose blocks are full of such tokens."""
    cache = torch.empty((num_blocks, hkv, sum(_sizes(d, bits))), dtype=torch.uint8, device="cuda")
    wide = torch.exp(0.5 * torch.randn((1, hkv, 1, d), generator=gen, device="cuda"))
    mean = torch.randn((1, hkv, 1, d), generator=gen, device="cuda")
    step = max(1, (1 << 26) // (hkv * d * BS))
    for a in range(0, num_blocks, step):
        n = min(step, num_blocks - a)
        k = torch.randn((n, hkv, BS, d), generator=gen, device="cuda") * wide + mean
        v = torch.randn((n, hkv, BS, d), generator=gen, device="cuda")
        _store(cache[a:a + n], k.bfloat16().float(), v.bfloat16().float(), d, bits)
    return cache


def prepare(case, seed):
    rng = np.random.default_rng(seed)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return {"append": _prepare_append, "park": _prepare_park, "restore": _prepare_restore,
            "decode": _prepare_decode, "prefill": _prepare_prefill}[case["kind"]](case, rng, gen)


def _prepare_append(case, rng, gen):
    cached = _strata(rng, case["seqs"], case["ctx_lo"], case["ctx_hi"])
    new = _strata(rng, case["seqs"], case["new_lo"], case["new_hi"])
    lens = cached + new
    tables, num_blocks = _tables(rng, lens)
    hkv, d, bits = case["hkv"], case["d"], case["bits"]
    t = int(new.sum())
    # keys and values are the last parts of one fused projection's rows
    kv = torch.empty((t, 2 * hkv, d), dtype=torch.bfloat16, device="cuda")
    kv[:, :hkv] = _keys(gen, t, hkv, d)
    kv[:, hkv:] = _randn(gen, t, hkv, d)
    # the blocks that hold new tokens, and each new token's place among them, for the plain form
    first, last = cached // BS, -(-lens // BS)
    of_seq = np.cumsum(last - first) - (last - first)
    seq = np.repeat(np.arange(len(new)), last - first)
    blk = np.arange(len(seq)) - of_seq[seq] + first[seq]
    row = np.repeat(np.arange(len(new)), new)
    pos = np.arange(t) - (np.cumsum(new) - new)[row] + cached[row]
    return dict(kind="append", d=d, bits=bits, cache=_cache(gen, num_blocks, hkv, d, bits), kv=kv,
                hkv=hkv, tables=_i32(tables), cached=_i32(cached), max_new=int(new.max()),
                cu=_i32(np.concatenate([[0], np.cumsum(new)])),
                touched=torch.from_numpy(tables[seq, blk].astype(np.int64)).cuda(),
                place=torch.from_numpy(of_seq[row] + pos // BS - first[row]).cuda(),
                slot=torch.from_numpy(pos % BS).cuda())


def _pairs(case, rng):
    """Blocks of one pool and of another, in random order, and the pools' sizes."""
    n = case["blocks"]
    nb = n + n // 8 + 1
    return _i32(np.stack([rng.permutation(nb)[:n], rng.permutation(nb)[:n]], axis=1)), nb


def _pool(gen, nb, hkv, d):
    k = _keys(gen, nb * BS, hkv, d).view(nb, BS, hkv, d // 8, 8).permute(0, 2, 3, 1, 4).contiguous()
    return k, _randn(gen, nb, hkv, d, BS)


def _prepare_park(case, rng, gen):
    hkv, d, bits = case["hkv"], case["d"], case["bits"]
    pairs, nb = _pairs(case, rng)
    k, v = _pool(gen, nb, hkv, d)
    cache = torch.zeros((nb, hkv, sum(_sizes(d, bits))), dtype=torch.uint8, device="cuda")
    return dict(kind="park", d=d, bits=bits, k_cache=k, v_cache=v, cache=cache, pairs=pairs)


def _prepare_restore(case, rng, gen):
    hkv, d, bits = case["hkv"], case["d"], case["bits"]
    pairs, nb = _pairs(case, rng)
    bf16 = dict(dtype=torch.bfloat16, device="cuda")
    return dict(kind="restore", d=d, bits=bits, cache=_cache(gen, nb, hkv, d, bits), pairs=pairs,
                k_cache=torch.zeros((nb, hkv, d // 8, BS, 8), **bf16),
                v_cache=torch.zeros((nb, hkv, d, BS), **bf16))


def _prepare_decode(case, rng, gen):
    lens = _strata(rng, case["seqs"], case["ctx_lo"], case["ctx_hi"])
    tables, num_blocks = _tables(rng, lens)
    hq, hkv, d, bits, b = case["hq"], case["hkv"], case["d"], case["bits"], case["seqs"]
    state = dict(kind="decode", d=d, bits=bits, cache=_cache(gen, num_blocks, hkv, d, bits),
                 q=_randn(gen, b, hq, d), tables=_i32(tables), lens=_i32(lens), max_len=int(lens.max()),
                 scale=1.0 / math.sqrt(d), out=torch.empty((b, hq, d), dtype=torch.bfloat16, device="cuda"),
                 lse=torch.empty((b, hq), device="cuda") if case["lse"] else None)
    if own:
        from paper_2607_23815_amd import lib
        state["ws"] = lib.alloc_workspace(lib.pkv_quant_decode_workspace_bytes(
            b, hq, hkv, d, bits, state["max_len"]))
    return state


def _prepare_prefill(case, rng, gen):
    cached = _strata(rng, case["seqs"], case["ctx_lo"], case["ctx_hi"])
    new = _strata(rng, case["seqs"], case["new_lo"], case["new_hi"])
    lens = cached + new
    tables, num_blocks = _tables(rng, lens)
    hq, hkv, d, bits = case["hq"], case["hkv"], case["d"], case["bits"]
    t = int(new.sum())
    state = dict(kind="prefill", d=d, bits=bits, cache=_cache(gen, num_blocks, hkv, d, bits),
                 q=_randn(gen, t, hq, d), tables=_i32(tables), cached=_i32(cached),
                 cu=_i32(np.concatenate([[0], np.cumsum(new)])), max_new=int(new.max()),
                 max_total=int(lens.max()), scale=1.0 / math.sqrt(d),
                 out=torch.empty((t, hq, d), dtype=torch.bfloat16, device="cuda"),
                 lse=torch.empty((t, hq), device="cuda") if case["lse"] else None,
                 host=list(zip(cached.tolist(), new.tolist())))
    if own:
        from paper_2607_23815_amd import lib
        state["ws"] = lib.alloc_workspace(lib.pkv_quant_prefill_workspace_bytes(
            len(new), t, hq, hkv, d, bits, state["max_new"], state["max_total"]))
    return state


# ----------------------------------------------------------------------------------------
# one pass
# ----------------------------------------------------------------------------------------
def run(state):
    if own:
        return _own(state)
    return {"append": _plain_append, "park": _plain_park, "restore": _plain_restore,
            "decode": _plain_decode, "prefill": _plain_prefill}[state["kind"]](state)


def _own(s):
    from paper_2607_23815_amd import lib
    kind = s["kind"]
    if kind == "append":
        lib.pkv_quant_append(s["cache"], s["kv"][:, :s["hkv"]], s["kv"][:, s["hkv"]:], s["tables"],
                             s["cached"], s["cu"], s["max_new"])
        return _shown(s["cache"], s["d"], s["bits"])
    if kind == "park":
        lib.pkv_quant_blocks(s["k_cache"], s["v_cache"], s["cache"], s["pairs"])
        return _shown(s["cache"], s["d"], s["bits"])
    if kind == "restore":
        lib.pkv_dequant_blocks(s["cache"], s["k_cache"], s["v_cache"], s["pairs"])
        return s["k_cache"], s["v_cache"]
    if kind == "decode":
        lib.pkv_quant_decode_attention(s["cache"], s["q"], s["tables"], s["lens"], s["max_len"], s["scale"],
                                       s["out"], lse=s["lse"], workspace=s["ws"])
    else:
        lib.pkv_quant_prefill_attention(s["cache"], s["q"], s["tables"], s["cached"], s["cu"], s["max_new"],
                                        s["max_total"], s["scale"], s["out"], lse=s["lse"],
                                        workspace=s["ws"])
    return (s["out"], s["lse"]) if s["lse"] is not None else s["out"]


def _power(e):
    """2^e in 32 bits."""
    return (e.int() + 127 << 23).view(torch.float32)


def _rounded(y, bits):
    """Codes of |y| <= M, to nearest even."""
    if bits == 8:
        return y.to(torch.float8_e4m3fn).view(torch.uint8)
    m = y.abs()
    code = (m > 0.25).byte() + (m >= 0.75) + (m > 1.25) + (m >= 1.75) + (m > 2.5) + (m >= 3.5) + (m > 5)
    return code | torch.signbit(y).byte() << 3


def _quantised_keys(x, bits):
    """x [.., d] in 32 bits: codes [.., d] and scale bytes [.., d / 32]."""
    x = x.unflatten(-1, (-1, 32))
    top = x.abs().amax(-1, keepdim=True)
    live = (top >= 2.0 ** -100) & torch.isfinite(top)
    frac, exp = torch.frexp(torch.where(live, top, 1.0))  # top = frac 2^exp, 1/2 <= frac < 1
    over = frac > (0.875 if bits == 8 else 0.75)          # M = 7/8 2^9, 3/4 2^3
    e = (exp - (9 if bits == 8 else 3) + over).clamp(max=TOP[bits])
    y = (x * _power(-e)).clamp(-MOST[bits], MOST[bits])
    codes = torch.where(live, _rounded(torch.where(live, y, 0.0), bits), 0)
    byte = torch.where(live, e + 127, torch.where(torch.isfinite(top), 127, 255))
    return codes.flatten(-2), byte.squeeze(-1).byte()


def _quantised_values(x, bits):
    """x [.., d] in 32 bits: codes [.., d] and scales [..]."""
    top = x.abs().amax(-1, keepdim=True)
    live = (top >= 2.0 ** -100) & torch.isfinite(top)
    s = torch.where(live, top.double() / MOST[bits], 1.0).float()
    s = ((s.view(torch.int32) + 0xFFFFF) & -0x100000).view(torch.float32)  # up to 4 significant bits
    s = s.clamp(max=TOP_VALUE[bits])
    y = torch.where(live, x.double() / s, 0.0).clamp(-MOST[bits], MOST[bits]).float()
    codes = torch.where(live, _rounded(y, bits), 0)
    return codes, torch.where(torch.isfinite(top), s, float("nan")).squeeze(-1)


def _store(cache, k, v, d, bits):
    """Whole blocks k, v [blocks, hkv, 16, d] into cache."""
    kc, ke, vc, vs = _parts(cache, d, bits)
    codes, byte = _quantised_keys(k, bits)
    kc.copy_(_key_bytes(codes, d, bits))
    ke.copy_(byte)
    codes, scale = _quantised_values(v, bits)
    vc.copy_(_value_bytes(codes, d, bits))
    vs.copy_(scale)


def _loaded(cache, d, bits):
    """Blocks' keys and values [blocks, hkv, 16, d] in 32 bits."""
    kc, ke, vc, vs = _parts(cache, d, bits)
    scale = torch.where(ke == 255, float("nan"), _power(ke.int() - 127))
    k = _values(_key_codes(kc, bits), bits).unflatten(-1, (-1, 32)) * scale[..., None]
    return k.flatten(-2), _values(_value_codes(vc, bits), bits) * vs[..., None]


def _plain_append(s):
    """The touched blocks' codes with the new tokens' put in their places."""
    d, bits, hkv = s["d"], s["bits"], s["hkv"]
    part = s["cache"][s["touched"]]
    kc, ke, vc, vs = _parts(part, d, bits)
    at = (s["place"], slice(None), s["slot"])
    codes, byte = _quantised_keys(s["kv"][:, :hkv].float(), bits)
    keys = _key_codes(kc, bits)
    keys[at] = codes
    kc.copy_(_key_bytes(keys, d, bits))
    ke[at] = byte
    codes, scale = _quantised_values(s["kv"][:, hkv:].float(), bits)
    values = _value_codes(vc, bits)
    values[at] = codes
    vc.copy_(_value_bytes(values, d, bits))
    vs[at] = scale
    s["cache"][s["touched"]] = part
    return _shown(s["cache"], d, bits)


def _plain_park(s):
    src, dst = s["pairs"].long().unbind(1)
    k = s["k_cache"][src].float().permute(0, 1, 3, 2, 4).flatten(-2)
    part = s["cache"][dst]
    _store(part, k, s["v_cache"][src].float().transpose(-2, -1), s["d"], s["bits"])
    s["cache"][dst] = part
    return _shown(s["cache"], s["d"], s["bits"])


def _plain_restore(s):
    src, dst = s["pairs"].long().unbind(1)
    k, v = _loaded(s["cache"][src], s["d"], s["bits"])
    s["k_cache"][dst] = k.unflatten(-1, (-1, 8)).transpose(2, 3).bfloat16()
    s["v_cache"][dst] = v.transpose(-2, -1).bfloat16()
    return s["k_cache"], s["v_cache"]


def _attended(q, key, val, seen, scale):
    """q [.., n, d], key and val [.., keys, d], seen [.., n, keys]: outputs and log-sum-exps."""
    score = torch.matmul(q, key.transpose(-2, -1)) * scale
    score = torch.where(seen, score, -float("inf"))
    top = score.amax(-1, keepdim=True)
    weight = torch.exp(score - top)
    total = weight.sum(-1, keepdim=True)
    return torch.matmul(weight, val) / total, (top + torch.log(total)).squeeze(-1)


def _plain_decode(s):
    b, hq, d = s["q"].shape
    hkv = s["cache"].shape[1]
    width = s["tables"].shape[1]
    slot = torch.arange(width * BS, device="cuda")
    step = max(1, (1 << 28) // (hkv * width * BS * d))
    for a in range(0, b, step):  # (as many sequences as 1 GB of keys in 32 bits holds)
        ids = s["tables"][a:a + step].clamp(min=0).long()
        n = ids.shape[0]
        k, v = _loaded(s["cache"][ids].flatten(0, 1), d, s["bits"])
        k, v = (x.view(n, width, hkv, BS, d).transpose(1, 2).reshape(n, hkv, width * BS, d) for x in (k, v))
        seen = (slot < s["lens"][a:a + step, None]).view(n, 1, 1, -1)
        out, lse = _attended(s["q"][a:a + step].float().view(n, hkv, hq // hkv, d), k, v, seen, s["scale"])
        s["out"][a:a + step] = out.view(n, hq, d).bfloat16()
        if s["lse"] is not None:
            s["lse"][a:a + step] = lse.view(n, hq)
    return (s["out"], s["lse"]) if s["lse"] is not None else s["out"]


def _plain_prefill(s):
    t, hq, d = s["q"].shape
    hkv = s["cache"].shape[1]
    g = hq // hkv
    row = 0
    for i, (p, n) in enumerate(s["host"]):
        ids = s["tables"][i, :-(-(p + n) // BS)].long()
        k, v = _loaded(s["cache"][ids], d, s["bits"])
        k, v = (x.transpose(0, 1).reshape(hkv, -1, d)[:, :p + n] for x in (k, v))
        q = s["q"][row:row + n].float().view(n, hkv, g, d).permute(1, 2, 0, 3).reshape(hkv, g * n, d)
        at = torch.arange(p + n, device="cuda")
        seen = (at <= p + torch.arange(n, device="cuda")[:, None]).repeat(g, 1)
        out, lse = _attended(q, k, v, seen, s["scale"])
        s["out"][row:row + n] = out.view(hkv, g, n, d).permute(2, 0, 1, 3).reshape(n, hq, d).bfloat16()
        if s["lse"] is not None:
            s["lse"][row:row + n] = lse.view(hq, n).T
        row += n
    return (s["out"], s["lse"]) if s["lse"] is not None else s["out"]


# ----------------------------------------------------------------------------------------
# the definitions in 64 bits
# ----------------------------------------------------------------------------------------
def exact(case, seed):
    """Dim by dim and sequence by sequence, from the definitions; None where that would take long."""
    global own
    w = work(case)
    if w["bytes"] > 2.0e9 or w["flops"] > 1.0e12:
        return None
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return {"append": _exact_append, "park": _exact_park, "restore": _exact_restore,
            "decode": _exact_decode, "prefill": _exact_prefill}[case["kind"]](s)


def _grid(bits):
    """The values of the codes 0, 1, ... that are not negative, ascending."""
    if bits == 4:
        return torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device="cuda")
    # 3 bits behind the point, exponents from -6 on, the lowest without a leading one
    return torch.tensor([math.ldexp(c % 8 + (8 if c >= 8 else 0), max(c // 8, 1) - 10) for c in range(127)],
                        dtype=torch.float64, device="cuda")


def _nearest(y, bits):
    """The code next to y, of two as near the even one."""
    grid = _grid(bits)
    m = y.abs()
    up = torch.searchsorted(grid, m.contiguous()).clamp(1, len(grid) - 1)
    down = up - 1
    far_up, far_down = grid[up] - m, m - grid[down]
    code = torch.where((far_up < far_down) | ((far_up == far_down) & (up % 2 == 0)), up, down)
    return code + torch.signbit(y).long() * (len(grid) if bits == 4 else 128)


def _exact_power(e):
    return (e.long() + 1023 << 52).view(torch.float64)


def _exact_key_code(x, bits):
    """x [n, 32] in 64 bits: codes and bytes."""
    top = x.abs().amax(1)
    fine = torch.isfinite(x).all(1)
    held = fine & (top >= 2.0 ** -100)
    e = torch.frexp(torch.where(held, top, 1.0)).exponent.long()  # (M 2^e is above it)
    for _ in range(10):
        e = torch.where(MOST[bits] * _exact_power(e - 1) >= top, e - 1, e)
    e = torch.where(held, e.clamp(max=TOP[bits]), 0)
    y = torch.where(held[:, None], x * _exact_power(-e)[:, None], 0.0).clamp(-MOST[bits], MOST[bits])
    code = _nearest(y, bits)
    return torch.where(held[:, None], code, 0), torch.where(fine, e + 127, 255)


def _exact_value_code(x, bits):
    """x [n, d] in 64 bits: codes and scales."""
    top = x.abs().amax(1)
    fine = torch.isfinite(x).all(1)
    held = fine & (top >= 2.0 ** -100)
    frac, exp = torch.frexp(torch.where(held, top, 1.0) / MOST[bits])
    step = _exact_power(exp - 4)
    s = torch.ceil(frac * 16) * step
    s = torch.where((s - step) * MOST[bits] >= top, s - step, s)  # (the quotient was rounded up past s)
    s = s.clamp(max=TOP_VALUE[bits])
    y = (torch.where(held[:, None], x, 0.0) / s[:, None]).clamp(-MOST[bits], MOST[bits])
    code = torch.where(held[:, None], _nearest(y, bits), 0)
    return code, torch.where(fine, torch.where(held, s, 1.0), float("nan"))


def _exact_parts(s, nb, hkv, d, bits, tokens):
    """The outputs of a write: the cache's parts with tokens (block, slot, k, v [n, hkv, d]) in them."""
    k, e, v, sc = (x.clone() for x in _parts(s["cache"], d, bits))
    block, slot, kx, vx = tokens
    grid = _grid(8) if bits == 8 else None
    if bits == 8:
        k, v = k.view(torch.float8_e4m3fn).double(), v.view(torch.float8_e4m3fn).double()
    else:
        k, v = k.long(), v.long()
    e, sc = e.long(), sc.double()
    per = 16 * 8 // bits
    planes = v.shape[2]
    for h in range(hkv):
        codes, byte = _exact_key_code(kx[:, h].reshape(-1, 32).double(), bits)
        codes = codes.view(-1, d)
        e[block, h, slot] = byte.view(-1, d // 32)
        vcodes, scale = _exact_value_code(vx[:, h].double(), bits)
        sc[block, h, slot] = scale
        for c in range(d):
            a, b = c // 16, c % 16
            at_v = (block, h, a // (d // 16 // planes), slot // 4, b, a % (d // 16 // planes))
            if bits == 8:
                value = lambda x: torch.where(x >= 128, -1.0, 1.0) * grid[x % 128]  # noqa: E731
                k[block, h, c // per, slot, c % per] = value(codes[:, c])
                v[at_v + (slot % 4,)] = value(vcodes[:, c])
            else:
                shift = 4 * (c % 2)
                at = (block, h, c // per, slot, c % per // 2)
                k[at] = k[at] & ~(15 << shift) | codes[:, c] << shift
                for j in range(4):  # (tokens that share a byte are not written at once)
                    m = slot % 4 == j
                    at = tuple(x[m] if torch.is_tensor(x) else x for x in at_v) + (j // 2,)
                    v[at] = v[at] & ~(15 << 4 * (j % 2)) | vcodes[m, c] << 4 * (j % 2)
    return k, e, v, sc


def _exact_append(s):
    nb, hkv = s["cache"].shape[:2]
    tokens = s["touched"][s["place"]], s["slot"], s["kv"][:, :hkv], s["kv"][:, hkv:]
    return _exact_parts(s, nb, hkv, s["d"], s["bits"], tokens)


def _exact_park(s):
    nb, hkv = s["cache"].shape[:2]
    src, dst = s["pairs"][:, 0].long(), s["pairs"][:, 1].long()
    d = s["d"]
    k = torch.cat([s["k_cache"][src, :, :, t].reshape(-1, hkv, d) for t in range(BS)])
    v = torch.cat([s["v_cache"][src, :, :, t] for t in range(BS)])
    slot = torch.arange(BS, device="cuda").repeat_interleave(len(src))
    return _exact_parts(s, nb, hkv, d, s["bits"], (dst.repeat(BS), slot, k, v))


def _exact_tokens(cache, d, bits):
    """Keys and values [hkv, blocks * 16, d] in 64 bits, dim by dim from the slabs' bytes."""
    kc, ks, vc, _ = _sizes(d, bits)
    n, hkv = cache.shape[:2]
    grid = _grid(bits)
    table = torch.cat([grid, -grid]) if bits == 4 else torch.cat([grid, grid[:1], -grid, grid[:1]])
    per, run = 16 * 8 // bits, d // 16 // max(1, d * bits // 512)
    key = torch.empty((hkv, n, BS, d), dtype=torch.float64, device="cuda")
    val = torch.empty((hkv, n, BS, d), dtype=torch.float64, device="cuda")
    slabs = cache.transpose(0, 1).contiguous()
    scale = _exact_power(slabs[..., kc:kc + ks].long() - 127).view(hkv, n, BS, d // 32)
    weight = slabs[..., kc + ks + vc:].contiguous().view(torch.float32).double()
    slot = torch.arange(BS, device="cuda")

    def value(first, at):  # what code number `at` behind byte `first` stands for
        byte = slabs[..., first + at * bits // 8].long()
        return table[byte if bits == 8 else byte >> 4 * (at % 2) & 15]

    for c in range(d):
        key[..., c] = value(0, (c // per * BS + slot) * per + c % per) * scale[..., c // 32]
        a, b = c // 16, c % 16
        at = a // run * 64 * run * 4 + ((slot // 4 * 16 + b) * run + a % run) * 4 + slot % 4
        val[..., c] = value(kc + ks, at) * weight
    return key.flatten(1, 2), val.flatten(1, 2)


def _exact_restore(s):
    k_cache, v_cache = s["k_cache"].double(), s["v_cache"].double()
    src, dst = s["pairs"][:, 0].long(), s["pairs"][:, 1].long()
    hkv, d = s["cache"].shape[1], s["d"]
    k, v = _exact_tokens(s["cache"][src], d, s["bits"])
    for h in range(hkv):
        for c in range(d):
            k_cache[dst, h, c // 8, :, c % 8] = k[h, :, c].view(-1, BS)
            v_cache[dst, h, c] = v[h, :, c].view(-1, BS)
    return k_cache, v_cache


def _exact_rows(q, key, val, scale, seen):
    """Each row of q [n, d] over its first `seen` keys."""
    z = torch.mm(q, key.T.contiguous()) * scale
    z = z.masked_fill(torch.arange(key.shape[0], device="cuda") >= seen[:, None], -float("inf"))
    norm = torch.logsumexp(z, dim=1)
    return torch.mm(torch.exp(z - norm[:, None]), val), norm


def _exact_decode(s):
    b, hq, d = s["q"].shape
    g = hq // s["cache"].shape[1]
    out = torch.zeros((b, hq, d), dtype=torch.float64, device="cuda")
    lse = torch.zeros((b, hq), dtype=torch.float64, device="cuda")
    for i, n in enumerate(s["lens"].tolist()):
        k, v = _exact_tokens(s["cache"][s["tables"][i, :-(-n // BS)].long()], d, s["bits"])
        seen = torch.full((g,), n, device="cuda")
        for h in range(0, hq, g):
            out[i, h:h + g], lse[i, h:h + g] = _exact_rows(s["q"][i, h:h + g].double(), k[h // g], v[h // g],
                                                           s["scale"], seen)
    return (out, lse) if s["lse"] is not None else out


def _exact_prefill(s):
    t, hq, d = s["q"].shape
    g = hq // s["cache"].shape[1]
    out = torch.zeros((t, hq, d), dtype=torch.float64, device="cuda")
    lse = torch.zeros((t, hq), dtype=torch.float64, device="cuda")
    row = 0
    for i, (p, n) in enumerate(s["host"]):
        k, v = _exact_tokens(s["cache"][s["tables"][i, :-(-(p + n) // BS)].long()], d, s["bits"])
        seen = p + 1 + torch.arange(n, device="cuda")
        for h in range(hq):
            out[row:row + n, h], lse[row:row + n, h] = _exact_rows(s["q"][row:row + n, h].double(), k[h // g],
                                                                   v[h // g], s["scale"], seen)
        row += n
    return (out, lse) if s["lse"] is not None else out


# ----------------------------------------------------------------------------------------
# what a pass cannot do without
# ----------------------------------------------------------------------------------------
def work(case):
    """Each input read once and each output written once, at the mean of the drawn lengths; 16-bit rows,
    queries and outputs, and the cache's codes and scales."""
    hkv, d = case["hkv"], case["d"]
    narrow = sum(_sizes(d, case["bits"])) / BS * hkv  # bytes of a token
    wide = 4 * hkv * d
    if case["kind"] in ("park", "restore"):
        return {"bytes": case["blocks"] * (BS * (narrow + wide) + 8), "flops": 0}
    b = case["seqs"]
    ctx = b * (case["ctx_lo"] + case["ctx_hi"]) / 2
    if case["kind"] == "decode":
        rows = b * case["hq"]
        return {"bytes": ctx * narrow + rows * (4 * d + (4 if case["lse"] else 0)),
                "flops": 4 * ctx * case["hq"] * d}
    new = b * (case["new_lo"] + case["new_hi"]) / 2
    if case["kind"] == "append":
        return {"bytes": new * (narrow + wide), "flops": 0}
    rows = new * case["hq"]
    return {"bytes": (ctx + new) * narrow + rows * (4 * d + (4 if case["lse"] else 0)),
            "flops": 4 * rows * d * (ctx + new / 2) / b}
