"""GPU tier: the calls of the quantised cache one after the other, as a serving loop makes them: prompts appended
and prefilled, decode steps (append, then attention), a prefix parked from the bf16 pool and restored to it. What
each call leaves is checked against its definition in 64 bits on the bytes that the calls before it left; steps
captured in a graph are replayed with new tokens, lengths and tables, and against the same calls made eagerly."""
import numpy as np
import pytest

from oracle import quant as Q
from tests.gpu_util import bf16_to_f64, i32, say, to_dev_bits, to_host_bits
from tests.paged_fixture import rand_bf16
from tests.test_gpu_quant_attention import BS, parts_off, rows_of

pytestmark = pytest.mark.gpu


class Loop:
    """The arrays that a program keeps. Sequence i's blocks are row i of the tables; the last is padding."""

    def __init__(self, lib, heads, bits, seqs, longest, seed):
        import torch
        self.lib, (self.hq, self.hkv, self.d), self.bits = lib, heads, bits
        self.rng = np.random.default_rng(seed)
        self.seqs, self.longest = seqs, longest
        width = -(-longest // BS)
        self.num_blocks = seqs * width + 2
        self.tables_host = self.rng.permutation(self.num_blocks)[:seqs * width].reshape(seqs, width).astype(np.int32)
        self.tables = i32(self.tables_host)
        self.cache = lib.alloc_quant_cache(self.num_blocks, self.hkv, self.d, bits)
        self.cache.fill_(255)
        self.scale = self.d ** -0.5
        self.lens = np.zeros(seqs, np.int64)
        self.ws = lib.alloc_workspace(lib.pkv_quant_decode_workspace_bytes(seqs, self.hq, self.hkv, self.d, bits,
                                                                           longest))
        self.keys = [np.zeros((0, self.hkv, self.d)) for _ in range(seqs)]    # as they were appended
        self.values = [np.zeros((0, self.hkv, self.d)) for _ in range(seqs)]
        self.torch = torch

    def rows(self, n, heads):
        return rand_bf16(self.rng, (n, heads, self.d))

    def note(self, k, v, new):
        at = 0
        for i, n in enumerate(new):
            self.keys[i] = np.concatenate([self.keys[i], bf16_to_f64(k[at:at + n])])
            self.values[i] = np.concatenate([self.values[i], bf16_to_f64(v[at:at + n])])
            at += n

    def check_cache(self):
        """Every token's codes and scales are those of its own 32-dim groups and values."""
        host = self.cache.cpu().numpy()
        for i, n in enumerate(self.lens):
            if n == 0:
                continue
            k, v = Q.stands_for(host[self.tables_host[i, :-(-n // BS)]], self.d, self.bits)
            pad = -n % BS
            blocks = lambda x: np.pad(x, ((0, pad), (0, 0), (0, 0))).reshape(-1, BS, self.hkv, self.d).transpose(
                0, 2, 1, 3)
            want = Q.stands_for(Q.blocks(blocks(self.keys[i]), blocks(self.values[i]), self.d, self.bits), self.d,
                                self.bits)
            for got, w in zip((k, v), want):
                flat = lambda x: x.transpose(0, 2, 1, 3).reshape(-1, self.hkv, self.d)[:n]
                assert np.array_equal(flat(got), flat(w)), i
        return host

    def check_rows(self, host, q, out, lse, i, n, weight_off, parts):
        """Row q [hq][d] of sequence i, which sees n keys."""
        k, v = (x.transpose(1, 0, 2, 3).reshape(self.hkv, -1, self.d)[:, :n]
                for x in Q.stands_for(host[self.tables_host[i, :-(-n // BS)]], self.d, self.bits))
        g = self.hq // self.hkv
        for h in range(self.hkv):
            s = slice(h * g, h * g + g)
            x = bf16_to_f64(q[s])
            o, z, tol, tol_z = rows_of(x, k[h], v[h], self.scale, weight_off, parts_off(x, self.bits) if parts else 0.0)
            assert (np.abs(out[s] - o) <= tol).all() and (np.abs(lse[s] - z) <= tol_z).all(), (i, n, h)

    def prompts(self, new):
        torch, lib = self.torch, self.lib
        t = sum(new)
        fused = self.rows(t, self.hq + 2 * self.hkv)  # one projection's rows
        dev = to_dev_bits(fused)
        q, k, v = dev[:, :self.hq].contiguous(), dev[:, self.hq:self.hq + self.hkv], dev[:, self.hq + self.hkv:]
        cached, cu = i32(self.lens), i32(np.concatenate([[0], np.cumsum(new)]))
        lib.pkv_quant_append(self.cache, k, v, self.tables, cached, cu, max(new))
        out = torch.empty((t, self.hq, self.d), dtype=torch.bfloat16, device="cuda")
        lse = torch.empty((t, self.hq), device="cuda")
        total = int((self.lens + new).max())
        need = lib.pkv_quant_prefill_workspace_bytes(self.seqs, t, self.hq, self.hkv, self.d, self.bits, max(new), total)
        lib.pkv_quant_prefill_attention(self.cache, q, self.tables, cached, cu, max(new), total, self.scale, out, lse=lse,
                                        workspace=lib.alloc_workspace(need))
        self.note(fused[:, self.hq:self.hq + self.hkv], fused[:, self.hq + self.hkv:], new)
        before = self.lens.copy()
        self.lens += new
        host = self.check_cache()
        got, z, at = bf16_to_f64(to_host_bits(out)), lse.double().cpu().numpy(), 0
        for i, n in enumerate(new):
            for j in {0, n // 2, n - 1} if n else ():
                self.check_rows(host, fused[at + j, :self.hq], got[at + j], z[at + j], i, int(before[i]) + j + 1, 2.0**-8,
                                True)
            at += n

    def step(self, make):
        """A decode step of every sequence that has keys; make(k, v, q, cached, cu, lens) leaves outputs."""
        new = (self.lens > 0).astype(np.int64)
        t = int(new.sum())
        k, v, q = self.rows(self.seqs, self.hkv), self.rows(self.seqs, self.hkv), self.rows(self.seqs, self.hq)
        out, lse = make(k, v, q, self.lens, np.concatenate([[0], np.cumsum(new)]), self.lens + new)
        self.note(k[:t], v[:t], new)
        self.lens += new
        host = self.check_cache()
        got, z = bf16_to_f64(to_host_bits(out)), lse.double().cpu().numpy()
        for i, n in enumerate(self.lens):
            if n:
                self.check_rows(host, q[i], got[i], z[i], i, int(n), 2.0**-16, False)
            else:
                assert (got[i] == 0).all() and (z[i] == -np.inf).all()


HEADS = [(8, 2, 128), (12, 4, 64)]


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("heads", HEADS)
def test_serving_loop(gpu_lib, heads, bits):
    """Prompts, a second turn behind them, and decode steps replayed from one graph between which the host only writes
    new numbers; the last sequence has no keys."""
    import torch
    lib = gpu_lib
    say(f"[quant loop] {heads}, bits {bits}")
    loop = Loop(lib, heads, bits, 5, 5200, 11 + bits)
    loop.prompts([37, 1, 2600, 16, 0])
    loop.prompts([5, 200, 70, 0, 0])
    hq, hkv, d = heads
    bf = lambda *n: torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    i = lambda n: torch.zeros(n, dtype=torch.int32, device="cuda")
    k, v, q, out = bf(5, hkv, d), bf(5, hkv, d), bf(5, hq, d), bf(5, hq, d)
    lse, cached, cu, lens = torch.zeros(5, hq, device="cuda"), i(5), i(6), i(5)

    def calls(o, z):
        lib.pkv_quant_append(loop.cache, k, v, loop.tables, cached, cu, 1)
        lib.pkv_quant_decode_attention(loop.cache, q, loop.tables, lens, loop.longest, loop.scale, o, lse=z,
                                       workspace=loop.ws)

    def fill(*hosts):
        for to, x in zip((k, v, q, cached, cu, lens), hosts):
            to.copy_(to_dev_bits(x) if x.dtype == np.uint16 else i32(x))

    def eager(*hosts):
        fill(*hosts)
        calls(out, lse)
        torch.cuda.synchronize()
        return out, lse

    loop.step(eager)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls(out, lse)

    def replayed(*hosts):
        fill(*hosts)
        out.fill_(7)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        o, z = bf(5, hq, d), torch.zeros_like(lse)
        calls(o, z)  # (the same tokens again: the same codes)
        torch.cuda.synchronize()
        assert torch.equal(o.view(torch.int16), out.view(torch.int16)) and torch.equal(z, lse)
        return out, lse

    for _ in range(3):
        loop.step(replayed)


@pytest.mark.parametrize("bits", [4, 8])
def test_two_graphs_share_a_workspace(gpu_lib, bits):
    """A prefill with splits and a decode, captured apart with one workspace and replayed one after the other on
    another stream than the current one, give the eager results every time."""
    import torch
    lib = gpu_lib
    hq, hkv, d = 8, 2, 128
    loop = Loop(lib, (hq, hkv, d), bits, 3, 6000, 5)
    loop.prompts([5900, 3000, 20])
    cached, cu, lens = i32([5850, 2990, 0]), i32([0, 50, 60, 80]), i32([5900, 3000, 20])
    q = to_dev_bits(loop.rows(80, hq))
    need = max(lib.pkv_quant_prefill_workspace_bytes(3, 80, hq, hkv, d, bits, 50, 5900),
               lib.pkv_quant_decode_workspace_bytes(3, hq, hkv, d, bits, 6000))
    assert need > 0
    ws = lib.alloc_workspace(need)
    outs = [torch.empty((n, hq, d), dtype=torch.bfloat16, device="cuda") for n in (80, 3)]
    stream = torch.cuda.Stream()
    prefill = lambda o, s=None: lib.pkv_quant_prefill_attention(loop.cache, q, loop.tables, cached, cu, 50, 5900, 0.1, o,
                                                                workspace=ws, stream=s)
    decode = lambda o, s=None: lib.pkv_quant_decode_attention(loop.cache, q[:3], loop.tables, lens, 6000, 0.1, o,
                                                              workspace=ws, stream=s)
    want = []
    stream.wait_stream(torch.cuda.current_stream())
    for call, o in zip((prefill, decode), outs):
        call(o, stream)
        stream.synchronize()
        want.append(o.clone())
    graphs = []
    for call, o in zip((prefill, decode), outs):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=stream):
            call(o)
    for _ in range(3):
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            for g in graphs:
                g.replay()
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            assert torch.equal(o.view(torch.int16), w.view(torch.int16))


@pytest.mark.parametrize("bits", [4, 8])
def test_a_parked_prefix(gpu_lib, bits):
    """A prefix in the bf16 pool is parked, attended to where it is, restored, and parked again, which changes
    little or nothing; the bf16 calls on the restored blocks see what the quantised calls see."""
    import torch
    lib = gpu_lib
    rng = np.random.default_rng(bits)
    hq, hkv, d, blocks = 8, 4, 64, 20
    k = to_dev_bits(rand_bf16(rng, (blocks, hkv, d // 8, BS, 8)))
    v = to_dev_bits(rand_bf16(rng, (blocks, hkv, d, BS)))
    cache = lib.alloc_quant_cache(30, hkv, d, bits)
    cache.fill_(255)
    to = rng.permutation(30)[:blocks].astype(np.int32)
    pairs = np.stack([np.arange(blocks, dtype=np.int32), to], 1)
    lib.pkv_quant_blocks(k, v, cache, i32(pairs))
    n = blocks * BS - 3
    q = to_dev_bits(rand_bf16(rng, (1, hq, d)))
    a, b = (torch.empty((1, hq, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    lib.pkv_quant_decode_attention(cache, q, i32(to[None]), i32([n]), n, 0.125, a)
    k2, v2 = torch.zeros_like(k), torch.zeros_like(v)
    lib.pkv_dequant_blocks(cache, k2, v2, i32(pairs[:, ::-1].copy()))
    lib.pkv_decode_attention(k2, v2, q, i32(np.arange(blocks)[None]), i32([n]), n, 0.125, b)
    x, y = a.double(), b.double()
    # both are within (2^-16 .. 2^-8) of sum w |v| and half a step of the output: values are below 5 in magnitude here
    top = float(v2.double().abs().max())
    assert ((x - y).abs() <= 2.0**-8 * (2 * top + x.abs() + y.abs())).all()
    lib.pkv_quant_blocks(k2, v2, cache, i32(pairs))
    lib.pkv_dequant_blocks(cache, k, v, i32(pairs[:, ::-1].copy()))
    # What a key group stands for stays: its largest code is above M / 2 (or is M / 2, and becomes M with half the
    # scale). So do values of 4 bits: the scale is rounded up by 1/8 at most, the largest code is 6 for all of
    # 16/3 .. 6. With 8 bits the largest may be 416, whose scale can be a step lower, and the others are rounded once
    # more: by 2^-4, or half of the least code, 2^-10 of a scale that is at most 9/8 / 448 of the largest.
    assert torch.equal(k.view(torch.int16), k2.view(torch.int16))
    off = (v.double() - v2.double()).abs()
    assert (off <= (0 if bits == 4 else 2.0**-4 * v2.double().abs() + top * 2.0**-18)).all()


@pytest.mark.parametrize("bits", [4, 8])
def test_padded_batch(gpu_lib, bits):
    """Rows behind the last sequence: none is appended, and outputs there stay as they were."""
    import torch
    lib = gpu_lib
    hq, hkv, d = 8, 2, 128
    loop = Loop(lib, (hq, hkv, d), bits, 2, 100, 3)
    loop.prompts([40, 7])
    cached, cu = i32(loop.lens), i32([0, 5, 6])
    fused = to_dev_bits(loop.rows(16, hq + 2 * hkv))
    k, v, q = fused[:, :hkv], fused[:, hkv:2 * hkv], fused[:, 2 * hkv:].contiguous()
    exact = loop.cache.clone()
    lib.pkv_quant_append(exact, k[:6], v[:6], loop.tables, cached, cu, 5)
    lib.pkv_quant_append(loop.cache, k, v, loop.tables, cached, cu, 16)  # (a bound above every length, too)
    assert torch.equal(loop.cache, exact)
    outs = []
    for rows, most in ((6, 5), (16, 16)):
        out, lse = torch.full((rows, hq, d), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((rows, hq), 7.0,
                                                                                                   device="cuda")
        lib.pkv_quant_prefill_attention(loop.cache, q[:rows], loop.tables, cached, cu, most, 40 + most, 0.1, out, lse=lse)
        outs.append((out, lse))
    (a, za), (b, zb) = outs
    assert torch.equal(a.view(torch.int16), b[:6].view(torch.int16)) and torch.equal(za, zb[:6])
    assert (b[6:] == 7).all() and (zb[6:] == 7).all()


def test_two_streams_without_workspaces(gpu_lib):
    """Decodes on two streams at once, each with the binding's own workspace of its stream."""
    import torch
    lib = gpu_lib
    hq, hkv, d, bits = 8, 2, 128, 4
    loop = Loop(lib, (hq, hkv, d), bits, 2, 6000, 4)
    loop.prompts([5900, 2000])
    lens = i32(loop.lens)
    qs = [to_dev_bits(loop.rows(2, hq)) for _ in range(2)]
    outs = [[torch.empty_like(q) for _ in range(6)] for q in qs]
    want = []
    for q, o in zip(qs, outs):
        lib.pkv_quant_decode_attention(loop.cache, q, loop.tables, lens, 6000, 0.1, o[0])
        want.append(o[0].clone())
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for n in range(6):
        for s, q, o in zip(streams, qs, outs):
            lib.pkv_quant_decode_attention(loop.cache, q, loop.tables, lens, 6000, 0.1, o[n], stream=s)
    torch.cuda.synchronize()
    for o, w in zip(outs, want):
        assert all(torch.equal(x.view(torch.int16), w.view(torch.int16)) for x in o)
