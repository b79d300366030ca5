"""GPU tier: the calls of a step that reads its cache sparsely, one after the other as a serving loop
makes them: tables grown on the GPU, queries and keys turned and appended, the key bounds of the
blocks written, blocks chosen, attention over them. First the prompts (ragged, with padding rows),
then decode steps replayed from one captured graph without the host between. Every call's outputs are
checked against its definition in 64 bits on what the calls before it left on the GPU, with the
tolerances of the calls' own tests."""
import numpy as np
import pytest

from tests import test_gpu_bounds, test_gpu_rope, test_gpu_select, test_gpu_sparse, test_gpu_tables
from tests.gpu_util import bf16_to_f64, i32, say, to_dev_bits, to_host_bits
from tests.paged_fixture import rand_bf16

pytestmark = pytest.mark.gpu

BS = 16


class Loop:
    """The arrays that a program keeps, and one step on them."""

    def __init__(self, lib, heads, seqs, rows, num_blocks, width, sizes, max_len, seed):
        import torch
        self.lib, (self.hq, self.hkv, self.d) = lib, heads
        self.sink, self.recent, self.blocks = sizes
        self.max_len, self.rows = max_len, rows
        rng = self.rng = np.random.default_rng(seed)
        zeros = lambda *n, dt=torch.int32: torch.zeros(n, dtype=dt, device="cuda")
        bf = torch.bfloat16
        self.tables = torch.full((seqs, width), -1, dtype=torch.int32, device="cuda")
        self.cached, self.lens, self.new = zeros(seqs), zeros(seqs), zeros(seqs)
        self.free = i32(rng.permutation(num_blocks))
        self.used, self.cu, self.status = zeros(1), zeros(seqs + 1), zeros(1)
        nan = lambda *n: to_dev_bits(np.full(n, 0x7FC0, np.uint16))
        self.k_cache = nan(num_blocks, self.hkv, self.d // 8, BS, 8)
        self.v_cache = nan(num_blocks, self.hkv, self.d, BS)
        self.bounds = nan(num_blocks, self.hkv, 2, self.d)
        self.axes = 3
        self.inv_freq = [1e4 ** (-j / 16) for j in range(16)]  # (half of the dims at D = 64)
        self.axis_of = [j % 3 for j in range(16)]
        self.rope = lib.rope_spec(self.inv_freq, axis_of=self.axis_of)
        self.size(rows)

    def size(self, rows):
        """Arrays of a step of up to `rows` rows."""
        import torch
        self.rows = rows
        zeros = lambda *n, dt=torch.int32: torch.zeros(n, dtype=dt, device="cuda")
        self.qkv = zeros(rows, self.hq + 2 * self.hkv, self.d, dt=torch.bfloat16)
        self.slots, self.row_seq = zeros(rows, dt=torch.int64), zeros(rows)
        self.positions, self.row_lens = zeros(self.axes, rows), zeros(rows)
        self.q = zeros(rows, self.hq, self.d, dt=torch.bfloat16)
        self.sel = zeros(rows, self.hkv, self.blocks)
        self.out = zeros(rows, self.hq, self.d, dt=torch.bfloat16)
        self.lse = zeros(rows, self.hq, dt=torch.float32)
        lib = self.lib
        self.ws = [lib.alloc_workspace(n) for n in (
            lib.pkv_select_workspace_bytes(rows, self.hq, self.hkv, self.d, self.max_len,
                                           self.blocks),
            lib.pkv_sparse_workspace_bytes(rows, self.hq, self.hkv, self.d, self.blocks))]

    def draw(self, new):
        self.new_host = np.asarray(new)
        self.new.copy_(i32(self.new_host))
        self.qkv.copy_(to_dev_bits(rand_bf16(self.rng, tuple(self.qkv.shape))))

    def step(self, max_new):
        lib = self.lib
        lib.pkv_extend_tables(self.tables, self.cached, self.new, self.free, self.used, self.used,
                              self.cu, self.lens, self.status, self.rows, slot_map=self.slots,
                              row_seq=self.row_seq, positions=self.positions[0],
                              row_lens=self.row_lens)
        self.positions[1:] = self.positions[0] // 7  # (a grid of images, say)
        q, k, v = self.qkv.split([self.hq, self.hkv, self.hkv], dim=1)
        lib.pkv_rope_append(self.k_cache, self.v_cache, q, k, v, self.slots, self.positions,
                            self.rope, self.q)
        lib.pkv_block_bounds(self.k_cache, self.v_cache, self.bounds, self.tables, self.cached,
                             self.cu, max_new)
        lib.pkv_select_blocks(self.bounds, self.q, self.tables, self.row_lens, self.max_len,
                              self.sink, self.recent, self.sel, row_seq=self.row_seq,
                              workspace=self.ws[0])
        lib.pkv_sparse_attention(self.k_cache, self.v_cache, self.q, self.tables, self.row_lens,
                                 self.sel, 0.125, self.out, row_seq=self.row_seq, lse=self.lse,
                                 workspace=self.ws[1])
        self.cached.copy_(self.lens)

    def state(self):
        h = lambda t: t.cpu().numpy().copy()
        return dict(tables=h(self.tables), cached=h(self.cached), used=int(self.used),
                    bounds=to_host_bits(self.bounds), pk=to_host_bits(self.k_cache),
                    pv=to_host_bits(self.v_cache), q=to_host_bits(self.q),
                    out=to_host_bits(self.out))

    def check(self, was):
        """This step's outputs, from the state before it."""
        now = self.state()
        new = self.new_host
        want, bits = test_gpu_tables.expect(was["tables"], was["cached"], new,
                                            self.free.cpu().numpy(), was["used"], self.rows)
        assert bits == 0 and int(self.status) == 0
        for got, k in ((now["tables"], "tables"), (now["used"], "used"), (now["cached"], "lens"),
                       (self.slots, "slots"), (self.row_seq, "seqs"), (self.positions[0], "pos"),
                       (self.row_lens, "row_lens")):
            got = got if isinstance(got, (int, np.ndarray)) else got.cpu().numpy()
            assert np.array_equal(got, want[k]), k
        n = int(new.sum())
        slots, hq, hkv, d = want["slots"][:n], self.hq, self.hkv, self.d
        # keys, values and queries
        pos = np.stack([want["pos"][:n]] + [want["pos"][:n] // 7] * 2)
        qkv = bf16_to_f64(to_host_bits(self.qkv))[:n]
        y, err = test_gpu_rope.turn(qkv, pos, self.axis_of, self.inv_freq, False, 1.0)
        test_gpu_rope.close(now["q"][:n], y[:, :hq], err[:, :hq], "q")
        rows_k = now["pk"][slots // BS, :, :, slots % BS].reshape(n, hkv, d)
        test_gpu_rope.close(rows_k, y[:, hq:hq + hkv], err[:, hq:hq + hkv], "k")
        rows_v = now["pv"][slots // BS, :, :, slots % BS]
        assert np.array_equal(bf16_to_f64(rows_v), qkv[:, hq + hkv:])
        assert np.array_equal(now["q"][n:], was["q"][n:]) and \
            np.array_equal(now["out"][n:], was["out"][n:]), "padding rows"
        # bounds, from the keys in the pool
        seqs = list(zip(was["cached"], new))
        test_gpu_bounds.check(now["bounds"], now["pk"], now["tables"], was["bounds"], seqs)
        # the choice, from these bounds and queries
        sel, seq = self.sel.cpu().numpy(), want["seqs"][:n]
        b64, q64 = bf16_to_f64(now["bounds"]), bf16_to_f64(now["q"])
        for t in range(n):
            want_sel = test_gpu_select.choice(b64, q64[t], now["tables"][seq[t]],
                                              want["row_lens"][t], self.sink, self.recent,
                                              self.blocks)
            assert np.array_equal(sel[t], want_sel), t
        # and the attention over it
        test_gpu_sparse.check((now["out"][:n], self.lse.cpu().numpy()[:n]), now["tables"],
                              now["pk"], now["pv"], now["q"][:n], want["row_lens"][:n], sel[:n],
                              0.125, seq)


@pytest.mark.parametrize("heads", [(8, 2, 64), (4, 4, 64), (16, 1, 128)])
def test_prompts_then_a_captured_decode_loop(gpu_lib, heads):
    import torch
    lib = gpu_lib
    say(f"[step] {heads[0]}/{heads[1]} heads of {heads[2]}")
    prompts = np.array([37, 0, 130, 300, 16, 5])
    loop = Loop(lib, heads, seqs=6, rows=500, num_blocks=64, width=24, sizes=(1, 2, 5),
                max_len=24 * BS, seed=heads[0])
    was = loop.state()
    loop.draw(prompts)
    loop.step(300)
    torch.cuda.synchronize()
    loop.check(was)

    loop.size(6)
    new = np.array([1, 1, 1, 1, 0, 1])  # one sequence has ended
    loop.draw(new)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            loop.step(1)
    for k in range(20):  # (past a block's end for every sequence)
        was = loop.state()
        loop.draw(new if k < 12 else np.array([0, 1, 1, 0, 0, 1]))
        graph.replay()
        torch.cuda.synchronize()
        if k % 4 == 0 or k == 15:
            loop.check(was)
        if k == 5:  # a full table refuses the whole step: nothing changes
            was = loop.state()
            keep = loop.cached.clone()
            loop.cached[3] = 24 * BS
            loop.draw(new)
            graph.replay()
            torch.cuda.synchronize()
            assert int(loop.status) == lib.PKV_EXTEND_TABLE_FULL
            loop.cached.copy_(keep)
            now = loop.state()
            for name in was:
                assert np.array_equal(was[name], now[name]), name


def test_sparse_rows_of_a_decode_step_without_row_seq(gpu_lib):
    """With one token per sequence the rows are the sequences: the same choice and outputs."""
    import torch
    lib = gpu_lib
    loop = Loop(lib, (8, 2, 64), seqs=4, rows=600, num_blocks=64, width=24, sizes=(1, 2, 5),
                max_len=24 * BS, seed=3)
    loop.draw([200, 33, 90, 250])
    loop.step(250)
    loop.size(4)
    loop.draw([1, 1, 1, 1])
    loop.step(1)
    sel, out = torch.zeros_like(loop.sel), torch.zeros_like(loop.out)
    lib.pkv_select_blocks(loop.bounds, loop.q, loop.tables, loop.lens, 24 * BS, 1, 2, sel)
    lib.pkv_sparse_attention(loop.k_cache, loop.v_cache, loop.q, loop.tables, loop.lens, sel, 0.125,
                             out)
    torch.cuda.synchronize()
    assert torch.equal(sel, loop.sel) and torch.equal(out.view(torch.int16),
                                                      loop.out.view(torch.int16))


def test_the_binding_refuses_wrong_tensors(gpu_lib):
    """Shapes, types, strides and devices that do not fit are refused before any launch."""
    import torch
    lib = gpu_lib
    loop = Loop(lib, (8, 2, 64), seqs=4, rows=4, num_blocks=8, width=4, sizes=(1, 2, 3), max_len=64,
                seed=1)
    q, k, v = loop.qkv.split([8, 2, 2], dim=1)
    rope = (loop.k_cache, loop.v_cache, q, k, v, loop.slots, loop.positions, loop.rope, loop.q)
    attend = (loop.k_cache, loop.v_cache, loop.q, loop.tables, loop.row_lens, loop.sel, 0.1, loop.out)
    select = (loop.bounds, loop.q, loop.tables, loop.row_lens, 64, 1, 2, loop.sel)
    bounds = (loop.k_cache, loop.v_cache, loop.bounds, loop.tables, loop.cached, loop.cu, 1)
    tables = (loop.tables, loop.cached, loop.new, loop.free, loop.used, loop.used, loop.cu, loop.lens,
              loop.status, 4)
    for call, args, which in (
            (lib.pkv_rope_append, rope, (0, 1, 2, 3, 4, 5, 6, 8)),
            (lib.pkv_sparse_attention, attend, (0, 1, 2, 3, 4, 5, 7)),
            (lib.pkv_select_blocks, select, (0, 1, 2, 3, 7)),
            (lib.pkv_block_bounds, bounds, (0, 1, 2, 3, 4, 5)),
            (lib.pkv_extend_tables, tables, (0, 1, 2, 3, 4, 5, 6, 7, 8))):
        for i in which:
            t = args[i]
            wide = torch.zeros(tuple(t.shape) + (2,), dtype=t.dtype, device="cuda")[..., 0]
            bads = [t.cpu(), t.float()]
            if t.numel() > 1:
                bads.append(wide)
            if t.dim() > 1:
                bads.append(t[None])
            if t.dtype == torch.bfloat16:
                bads.append(t[..., :-1].contiguous())
            for bad in bads:
                with pytest.raises((TypeError, ValueError)):
                    call(*args[:i], bad, *args[i + 1:])
                    say(f"  taken: {call.__name__} argument {i} as {bad.dtype} {tuple(bad.shape)}")
    with pytest.raises(ValueError):
        lib.pkv_rope_append(*rope[:6], loop.positions[0], *rope[7:])  # three axes are needed
