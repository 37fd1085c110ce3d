"""What the entry points of rotation, scored and shared attention hand to the library, and what they refuse before (no GPU needed)."""
import ctypes

import pytest
import torch

import paper_2608_23658_b200 as ekv
from test_binding_checks import a_pool, calls, gpu  # noqa: F401

BF16, I64 = torch.bfloat16, torch.int64


def pool_of(Hq=4, dtype=ekv.EKV_BF16):
    pool = a_pool()
    pool.num_q_heads, pool.block_size, pool.dtype, pool._parts, pool._ws = Hq, 16, dtype, {}, None
    return pool


def refused(call, good, bad):
    for name, values in bad.items():
        for v in values:
            with pytest.raises(ValueError):
                call(**{**good, name: v})


def test_rope_write_kv(calls):  # noqa: F811
    pool, T = pool_of(), 5
    rows = gpu(T, 10, 64, dtype=BF16)
    good = dict(layer=0, q=rows[:, :4], k=rows[:, 4:6], v=rows[:, 6:8], positions=gpu(T), inv_freq=gpu(16, dtype=torch.float32),
                slot_mapping=gpu(T, dtype=I64), q_weight=gpu(64, dtype=BF16), k_weight=None, q_out=gpu(T, 4, 64, dtype=BF16), stream=0)
    assert pool.rope_write_kv(**good) is good["q_out"]
    (name, handle, layer, rope, q, qs, k, ks, v, vs, out, outs, k_out, slots, n, stream), = calls
    assert (name, handle, layer, n, stream, qs, ks, vs, outs, k_out) == ("ekv_rope_write_kv", None, 0, T, 0, 640, 640, 640, 256, None)
    assert (q, k, v, out, slots) == tuple(good[x].data_ptr() for x in ("q", "k", "v", "q_out", "slot_mapping"))
    assert (rope.rotary_dim, rope.num_axes, rope.flags, rope.factor, rope.weight_offset) == (32, 1, 0, 1.0, 0.0)
    assert rope.positions == good["positions"].data_ptr() and rope.inv_freq == good["inv_freq"].data_ptr()
    assert rope.q_weight == good["q_weight"].data_ptr() and rope.k_weight is None and rope.pair_axis is None
    calls.clear()
    pool.rope_write_kv(**{**good, "positions": gpu(3, T), "axes": [0, 1, 2, 0] * 4, "interleaved": True})
    rope = calls[0][3]
    axes = ctypes.c_void_p.from_buffer(rope, ekv.Rope.pair_axis.offset).value
    assert rope.num_axes == 3 and rope.flags == ekv.EKV_ROPE_ADJACENT and ctypes.string_at(axes, 16) == bytes([0, 1, 2, 0] * 4)
    calls.clear()
    refused(pool.rope_write_kv, good, {
        "q": [rows[:, :3], rows[:4, :4], rows[:, :4].float(), torch.zeros(T, 4, 64, dtype=BF16), gpu(T, 64, 4, dtype=BF16).transpose(1, 2)],
        "k": [rows[:, 4:7], gpu(T, 2, 32, dtype=BF16)], "v": [rows[:, 6:7], gpu(T, 2, 64, dtype=torch.float16)],
        "q_out": [gpu(T, 2, 64, dtype=BF16), gpu(T, 4, 64)], "positions": [gpu(T - 1), gpu(T, dtype=I64), torch.zeros(T, dtype=torch.int32), gpu(3, T)],
        "inv_freq": [gpu(16), gpu(16, dtype=torch.float64)], "slot_mapping": [gpu(T), gpu(2 * T, dtype=I64)[::2]],
        "q_weight": [gpu(32, dtype=BF16), gpu(64, dtype=torch.float32)], "k_weight": [gpu(64)], "k_out": [gpu(T, 2, 64)]})
    assert not calls


def test_scored_attention(calls):  # noqa: F811
    pool, R, T = pool_of(), 3, 7
    ws = gpu(512, dtype=torch.uint8)
    decode = dict(layer=2, q=gpu(R, 4, 64, dtype=BF16), block_tables=gpu(R, 9), seq_lens=gpu(R), scale=0.5, cap=3.0, window=8, slopes=gpu(4, dtype=torch.float32),
                  prefix_lens=gpu(R), out=gpu(R, 4, 64, dtype=BF16), workspace=ws, stream=0)
    assert pool.attn_decode_scored(**decode) is decode["out"]
    name, handle, layer, q, out, tables, width, lens, n, scale, scores, at, size, stream = calls[0]
    assert (name, layer, width, n, scale, size, stream) == ("ekv_attn_decode_scored", 2, 9, R, 0.5, 512, 0)
    assert (scores.cap, scores.window, scores.slopes, scores.prefix_lens) == (3.0, 8, decode["slopes"].data_ptr(), decode["prefix_lens"].data_ptr())
    calls.clear()
    cu = torch.tensor([0, 1, 3, 7], dtype=torch.int32)
    prefill = dict(decode, q=gpu(T, 4, 64, dtype=BF16), out=gpu(T, 4, 64, dtype=BF16), cu_q_lens=gpu(R + 1), cu_q_lens_host=cu)
    pool.attn_prefill_chunk_scored(**prefill)
    assert calls[0][0] == "ekv_attn_prefill_chunk_scored" and calls[0][8] == cu.data_ptr() and calls[0][10] == R
    calls.clear()
    common = {"block_tables": [gpu(R, 9, dtype=I64), gpu(27), torch.zeros(R, 9, dtype=torch.int32), gpu(R + 1, 9)], "seq_lens": [gpu(R, dtype=I64)],
              "slopes": [gpu(5, dtype=torch.float32), gpu(4)], "prefix_lens": [gpu(R - 1), gpu(R, dtype=I64)]}
    refused(pool.attn_decode_scored, decode, {**common, "q": [gpu(R + 1, 4, 64, dtype=BF16), gpu(R, 4, 64)], "out": [gpu(R, 4, 64), gpu(R, 2, 64, dtype=BF16)]})
    refused(pool.attn_prefill_chunk_scored, prefill, {**common, "q": [gpu(T - 1, 4, 64, dtype=BF16)], "cu_q_lens": [gpu(R), gpu(R + 1, dtype=I64)],
                                                      "cu_q_lens_host": [cu[:3], cu.long(), torch.tensor([0, 1, 3, 8], dtype=torch.int32)]})
    assert not calls


def test_shared_decode(calls):  # noqa: F811
    pool, R = pool_of(), 5
    starts, shared = torch.tensor([0, 3, 5], dtype=torch.int32), torch.tensor([32, 0], dtype=torch.int32)
    good = dict(layer=0, q=gpu(R, 4, 64, dtype=BF16), block_tables=gpu(R, 9), seq_lens=gpu(R), group_starts=starts, shared_lens=shared, scale=0.5,
                out=gpu(R, 4, 64, dtype=BF16), workspace=gpu(512, dtype=torch.uint8), stream=0)
    pool.attn_decode_shared(**good)
    name, _, _, q, out, tables, width, lens, n, at_starts, at_shared, G, *rest = calls[0]
    assert (name, width, n, at_starts, at_shared, G) == ("ekv_attn_decode_shared", 9, R, starts.data_ptr(), shared.data_ptr(), 2)
    calls.clear()
    refused(pool.attn_decode_shared, good, {"group_starts": [starts.long(), starts[:2]], "shared_lens": [shared.float(), shared[:1]],
                                            "seq_lens": [gpu(R + 1), gpu(R, dtype=I64)], "q": [gpu(R, 4, 32, dtype=BF16)]})
    assert not calls


def test_the_library_refuses_null_pools_and_says_why():
    lib = ekv.load_library()
    rope, scores = ekv.Rope(), ekv.Scores()
    assert lib.ekv_rope_write_kv(None, 0, ctypes.byref(rope), *[0] * 10, 0, 0) == ekv.Status.ERR_INVALID
    assert lib.ekv_attn_decode_scored(None, 0, 0, 0, 0, 1, 0, 1, 1.0, ctypes.byref(scores), 0, 0, 0) == ekv.Status.ERR_INVALID
    assert lib.ekv_attn_prefill_chunk_scored(None, 0, 0, 0, 0, 1, 0, 0, 0, 1, 1.0, ctypes.byref(scores), 0, 0, 0) == ekv.Status.ERR_INVALID
    assert lib.ekv_attn_decode_shared(None, 0, 0, 0, 0, 1, 0, 1, 0, 0, 1, 1.0, 0, 0, 0) == ekv.Status.ERR_INVALID
    assert "NULL" in ekv.ekv_last_error()
    assert lib.ekv_attn_prefill_scored_workspace_bytes(None) == 0 and lib.ekv_attn_decode_shared_workspace_bytes(None, 0, 0, 0, 1) == 0
