"""Outputs that a call makes for its caller belong to the stream that writes them: memory that a kernel under way elsewhere may still use is not theirs."""
import pytest
import torch

import paper_2608_23658_b200 as ekv
from scored_model import DEV, Batch

pytestmark = pytest.mark.gpu


def owner(t):
    """The stream whose memory a tensor stands in."""
    at = t.data_ptr()
    stream, = [s["stream"] for s in torch.cuda.memory_snapshot() if s["address"] <= at < s["address"] + s["total_size"]]
    return stream


def every_call(b, **more):
    starts, shared = torch.tensor([0, 2], dtype=torch.int32), torch.tensor([0], dtype=torch.int32)
    last = (b.cu[1:] - 1).long()
    slots, inv_freq, first = torch.arange(b.T, device=DEV), torch.ones(32, device=DEV), b.tables[0, 0].long() * 16 + torch.arange(16, device=DEV)
    positions = slots.int()
    k = torch.zeros((b.T, 2, 64), dtype=torch.bfloat16, device=DEV)
    spare = ekv.Pool(num_q_heads=8, num_kv_heads=2, head_dim=64, base_blocks=40)
    q = b.q[last]
    return {
        "rope_write_kv": lambda: spare.rope_write_kv(0, b.q, k, k, positions, inv_freq, slots, **more),
        "attn_decode_scored": lambda: b.pool.attn_decode_scored(0, q, b.tables, b.seq_lens, b.scale, cap=9.0, **more),
        "attn_prefill_chunk_scored": lambda: b.pool.attn_prefill_chunk_scored(0, b.q, b.tables, b.cu, b.cu_host, b.seq_lens, b.scale, cap=9.0, **more),
        "attn_decode_shared": lambda: b.pool.attn_decode_shared(0, q, b.tables, b.seq_lens, starts, shared, b.scale, **more),
        "attn_decode": lambda: b.pool.attn_decode(0, q, b.tables, b.seq_lens, b.scale, **more),
        "attn_prefill_chunk": lambda: b.pool.attn_prefill_chunk(0, b.q, b.tables, b.cu, b.cu_host, b.seq_lens, b.scale, **more),
        "read_kv": lambda: b.pool.read_kv(0, first, **more)[1],
    }


@pytest.mark.parametrize("call", ["rope_write_kv", "attn_decode_scored", "attn_prefill_chunk_scored", "attn_decode_shared", "attn_decode",
                                  "attn_prefill_chunk", "read_kv"])
def test_an_output_belongs_to_the_stream_of_its_call(call):
    b, side = Batch(8, 2, 64, [300, 40], [50, 30], seed=51), torch.cuda.Stream()
    want = every_call(b)[call]()
    assert owner(want) == torch.cuda.current_stream().cuda_stream
    torch.cuda.synchronize()
    for stream in (side, side.cuda_stream):
        run = every_call(b, stream=stream)[call]
        torch.cuda.synchronize()
        out = run()
        torch.cuda.synchronize()
        assert owner(out) == side.cuda_stream and torch.equal(out, want)
