"""The workspace of a call that brings none belongs to the stream that the call runs on. It is dropped
as the call returns, with its kernels perhaps still to run, so its memory may only go on to work behind
them: memory of another stream would be handed out and written at once."""
from types import SimpleNamespace

import numpy as np
import pytest

HQ, HKV, D, ROWS = 4, 2, 64, 3


def calls(lib, device):
    """The calls that make a workspace of their own: (call, arguments, keyword arguments)."""
    import torch
    bf = lambda *n: torch.zeros(n, dtype=torch.bfloat16, device=device)
    i32 = lambda *n: torch.zeros(n, dtype=torch.int32, device=device)
    k, v = bf(8, HKV, D // 8, 16, 8), bf(8, HKV, D, 16)
    q, out, tables, lens = bf(ROWS, HQ, D), bf(ROWS, HQ, D), i32(ROWS, 4), i32(ROWS)
    cu, sel, bounds = i32(ROWS + 1), i32(ROWS, HKV, 2), bf(8, HKV, 2, D)
    return [
        (lib.pkv_decode_attention, (k, v, q, tables, lens, 64, 0.1, out)),
        (lib.pkv_mixed_attention, (k, v, 0.1, q, tables, lens, cu, 1, 64, out, q, tables, lens, 64, out)),
        (lib.pkv_select_blocks, (bounds, q, tables, lens, 64, 0, 1, sel)),
        (lib.pkv_sparse_attention, (k, v, q, tables, lens, sel, 0.1, out))]


@pytest.mark.parametrize("which", range(4))
def test_allocated_under_the_calls_stream(monkeypatch, which):
    import torch
    from paper_2607_23815_amd import lib
    current, made = [], []

    class Under:
        def __init__(self, stream):
            self.stream = stream

        def __enter__(self):
            current.append(self.stream)

        def __exit__(self, *_):
            current.pop()

    def alloc(nbytes, device="cuda"):
        made.append((nbytes, list(current)))

    stub = {n: lambda *_: 0 for n in ("pkv_decode_attention", "pkv_mixed_attention", "pkv_select_blocks",
                                      "pkv_sparse_attention")}
    stub.update({n: lambda *_: 4096 for n in ("pkv_decode_workspace_bytes", "pkv_select_workspace_bytes",
                                              "pkv_sparse_workspace_bytes")})
    lib._get_torch()
    monkeypatch.setattr(torch.cuda, "stream", Under)
    monkeypatch.setattr(lib, "alloc_workspace", alloc)
    monkeypatch.setattr(lib, "_lib", SimpleNamespace(**stub))
    monkeypatch.setattr(lib, "_dev_ptr", lambda *_: 0)
    monkeypatch.setattr(lib, "_ptr", lambda *_: 0)
    monkeypatch.setattr(lib, "_launch_on", lambda s: (0, 0))
    monkeypatch.setattr(lib, "_stream", lambda s: 0)
    call, args = calls(lib, "cpu")[which]
    side = SimpleNamespace(cuda_stream=1)
    call(*args, stream=side)
    assert made == [(4096, [side])]
    call(*args)
    assert made[1:] == [(4096, [])]
    call(*args, stream=side, workspace=torch.zeros(4096, dtype=torch.uint8))
    assert len(made) == 2


@pytest.mark.gpu
def test_memory_of_the_current_stream_is_not_taken(gpu_lib):
    """A choice and an attention in splits on a side stream that is behind, none with a workspace: what
    the current stream allocates and writes meanwhile changes nothing of their results."""
    import torch
    from tests import test_gpu_select, test_gpu_sparse
    from tests.gpu_util import i32, to_dev_bits, to_host_bits
    from tests.paged_fixture import rand_bf16
    lib = gpu_lib
    rng = np.random.default_rng(0)
    lens = np.array([16 * 700, 16 * 650 + 3])
    tables, pk, pv = test_gpu_sparse.pools(rng, list(lens), HKV, D)
    bounds = test_gpu_select.pool(rng, list(lens), HKV, D, nan=False)[1]
    q = rand_bf16(rng, (2, HQ, D))
    blocks = 200
    assert lib.pkv_select_workspace_bytes(2, HQ, HKV, D, int(lens.max()), blocks) > 0
    need = lib.pkv_sparse_workspace_bytes(2, HQ, HKV, D, blocks)
    assert need > 0
    dk, dv, dq, dt, dl, db = (to_dev_bits(pk), to_dev_bits(pv), to_dev_bits(q), i32(tables), i32(lens),
                              to_dev_bits(bounds))
    sel = torch.zeros((2, HKV, blocks), dtype=torch.int32, device="cuda")
    out = torch.zeros((2, HQ, D), dtype=torch.bfloat16, device="cuda")
    x = torch.randn((4096, 4096), device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(20):
            x = (x @ x).clamp_(-1, 1)
    lib.pkv_select_blocks(db, dq, dt, dl, int(lens.max()), 1, 2, sel, stream=side)
    lib.pkv_sparse_attention(dk, dv, dq, dt, dl, sel, 0.125, out, stream=side)
    kept = [torch.full((n,), 255, dtype=torch.uint8, device="cuda")
            for n in (need, 2 * need, 1 << 16, 1 << 18) for _ in range(8)]
    torch.cuda.synchronize()
    assert all(int(t.min()) == 255 for t in kept)
    got = sel.cpu().numpy()
    test_gpu_select.check(got, tables, bounds, q, lens, 1, 2, blocks)
    test_gpu_sparse.check((to_host_bits(out), None), tables, pk, pv, q, lens, got, 0.125)
