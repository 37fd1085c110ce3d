"""The free functions of rotation, scored and shared attention, which take a pool's handle: what they hand on, and what they refuse because the library would
read it on the host."""
import ctypes

import pytest
import torch

import paper_2608_23658_b200 as ekv
from test_binding_checks import calls, gpu  # noqa: F401

BF16, I32 = torch.bfloat16, torch.int32


def i32(*x):
    return torch.tensor(x, dtype=I32)


def test_what_the_library_reads_on_the_host_has_to_be_there(calls):  # noqa: F811
    R, q, tables, lens, scores = 3, gpu(7, 4, 64, dtype=BF16), gpu(3, 9), gpu(3), ekv.Scores(3.0, 0, None, None)
    prefill = lambda cu: ekv.ekv_attn_prefill_chunk_scored(5, 0, q, q, tables, gpu(R + 1), cu, lens, 0.5, scores, None, stream=0)
    shared = lambda starts, n: ekv.ekv_attn_decode_shared(5, 0, q, q, tables, lens, starts, n, 0.5, None, stream=0)
    size = lambda starts, n: ekv.ekv_attn_decode_shared_workspace_bytes(5, starts, n, 9)
    prefill(i32(0, 1, 3, 7))
    assert calls[0][0] == "ekv_attn_prefill_chunk_scored" and calls[0][10] == R
    for bad in (gpu(R + 1), i32(0, 1, 3), i32(0, 1, 3, 7).long(), i32(0, 9, 1, 9, 3, 9, 7, 9)[::2]):
        with pytest.raises(ValueError):
            prefill(bad)
    shared(i32(0, 2, 3), i32(32, 0)), size(i32(0, 2, 3), i32(32, 0))
    assert [c[0] for c in calls[1:]] == ["ekv_attn_decode_shared", "ekv_attn_decode_shared_workspace_bytes"]
    calls.clear()
    for starts, n in ((i32(0, 3), i32(32, 0)), (gpu(3), i32(32, 0)), (i32(0, 2, 3), gpu(2)), (i32(0, 2, 3).long(), i32(32, 0)), (i32(0, 2, 3), torch.zeros(2))):
        for call in (shared, size):
            with pytest.raises(ValueError):
                call(starts, n)
    assert not calls


@pytest.mark.gpu
def test_they_do_what_the_pool_does():
    from scored_model import DEV, Batch
    b = Batch(8, 2, 64, [5011, 800, 64], [1, 1, 1], seed=81)
    h, ws = b.pool.handle, torch.empty(1 << 26, dtype=torch.uint8, device=DEV)
    scores, out = ekv.Scores(9.0, 700, None, None), torch.empty_like(b.q)
    ekv.ekv_attn_decode_scored(h, 0, b.q, out, b.tables, b.seq_lens, b.scale, scores, ws)
    assert torch.equal(out, b.pool.attn_decode_scored(0, b.q, b.tables, b.seq_lens, b.scale, cap=9.0, window=700))
    ekv.ekv_attn_prefill_chunk_scored(h, 0, b.q, out, b.tables, b.cu, b.cu_host, b.seq_lens, b.scale, scores, ws)
    assert torch.equal(out, b.pool.attn_prefill_chunk_scored(0, b.q, b.tables, b.cu, b.cu_host, b.seq_lens, b.scale, cap=9.0, window=700))
    starts, shared = i32(0, 3), i32(0)
    ekv.ekv_attn_decode_shared(h, 0, b.q, out, b.tables, b.seq_lens, starts, shared, b.scale, ws)
    assert torch.equal(out, b.pool.attn_decode_shared(0, b.q, b.tables, b.seq_lens, starts, shared, b.scale))
    rows = torch.randn((3, 12, 64), device=DEV).to(BF16)
    positions, inv_freq, slots = torch.arange(3, dtype=I32, device=DEV), torch.rand(32, device=DEV), torch.arange(3, device=DEV)
    q, k, v = rows[:, :8], rows[:, 8:10], rows[:, 10:]
    rope = ekv.Rope(64, 1, 0, 1.0, 1e-6, 0.0, inv_freq.data_ptr(), positions.data_ptr(), None, None, None)
    assert ctypes.sizeof(rope) == 64
    ekv.ekv_rope_write_kv(h, 0, rope, q.data_ptr(), q.stride(0), k.data_ptr(), k.stride(0), v.data_ptr(), v.stride(0), out.data_ptr(), 8 * 64, None, slots.data_ptr(), 3)
    written = [x.clone() for x in b.pool.read_kv(0, slots)]
    assert torch.equal(out, b.pool.rope_write_kv(0, q, k, v, positions, inv_freq, slots))
    assert all(torch.equal(x, y) for x, y in zip(written, b.pool.read_kv(0, slots))) and b.pool.poll_status() == ekv.Status.OK
