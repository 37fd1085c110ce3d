"""Decode attention with capped, biased and windowed scores and visible prefixes against the model in 64 bits."""
import pytest
import torch

import paper_2608_23658_b200 as ekv
from scored_model import BF16, DEV, Batch, check, slopes_of

pytestmark = pytest.mark.gpu
LAYOUTS = [(4, 2, 64), (28, 4, 128), (8, 8, 64), (6, 2, 128), (5, 1, 64), (64, 8, 128)]
MODS = [{}, {"cap": 30.0}, {"window": 37}, {"bias": True}, {"prefix": 21}, {"cap": 5.0, "window": 300, "bias": True, "prefix": 18}, {"window": 1},
        {"window": 16, "prefix": 16}, {"cap": 50.0, "bias": True}, {"window": 5000, "prefix": 1000}]


def run(b, cap=0.0, window=0, bias=False, prefix=0, scale=None, **more):
    n = len(b.lens)
    slopes = slopes_of(b.Hq) if bias else None
    pre = torch.full((n,), prefix, dtype=torch.int32, device=DEV) if isinstance(prefix, int) else torch.tensor(prefix, dtype=torch.int32, device=DEV)
    use = pre if isinstance(prefix, list) or prefix else None
    got = b.pool.attn_decode_scored(0, b.q, b.tables, b.seq_lens, b.scale if scale is None else scale, cap=cap, window=window, slopes=slopes,
                                    prefix_lens=use, **more)
    return got, b.model(scale=scale, cap=cap, window=window, slopes=slopes, prefix=None if use is None else pre.tolist())


@pytest.mark.parametrize("mods", MODS, ids=str)
@pytest.mark.parametrize("Hq,Hk,D", LAYOUTS)
def test_against_the_model(Hq, Hk, D, mods):
    lens = [1, 2, 15, 16, 17, 36, 37, 38, 300, 701, 64]
    b = Batch(Hq, Hk, D, [x - 1 for x in lens], [1] * len(lens), seed=Hq + D, magnitude=4.0 if "cap" in mods else 1.0)
    got, want = run(b, **mods)
    check(got, want, str(mods))
    assert b.pool.poll_status() == ekv.Status.OK


@pytest.mark.parametrize("mods", [{"cap": 20.0}, {"window": 4000, "prefix": 50}, {"bias": True, "window": 9000}], ids=str)
def test_long_sequences_in_many_ranges(mods):
    b = Batch(8, 2, 128, [20011, 5, 9999], [1] * 3, seed=5, magnitude=3.0, table_extra=40)
    got, want = run(b, **mods)
    check(got, want, str(mods))


def test_empty_sequences_prefixes_of_every_length_and_scales_of_any_sign():
    b = Batch(4, 2, 64, [0, 99, 99, 99, 99], [1] * 5, seed=2)
    b.seq_lens[0] = 0
    got, (want, bound) = run(b, window=10, prefix=[5, -3, 0, 200, 33])
    assert (got[0] == 0).all()
    check(got[1:], (want[1:], bound[1:]))
    for scale in (-0.2, 0.0):
        for cap in (0.0, 4.0):
            got, (want, bound) = run(b, cap=cap, scale=scale)
            check(got[1:], (want[1:], bound[1:]), f"scale {scale} cap {cap}")


def test_scores_far_beyond_the_cap():
    b = Batch(4, 2, 64, [200, 60], [1, 1], seed=3, magnitude=500.0)
    for cap in (1.0, 50.0):
        check(*run(b, cap=cap))


def test_caps_of_any_size_and_queries_of_zeros():
    b = Batch(4, 2, 64, [200, 60], [1, 1], seed=16, magnitude=20.0)
    for cap in (1e-42, 1e-30, 1e-3, 3e3, 1e6, 1e30):
        check(*run(b, cap=cap), str(cap))
    b.q.zero_()
    for cap in (1e-42, 1e-30, 50.0, 1e6):
        check(*run(b, cap=cap), str(cap))


def test_what_a_row_does_not_see_does_not_reach_it():
    b = Batch(4, 2, 128, [199, 150], [1, 1], seed=4)
    _, want = run(b, window=40, prefix=20)
    for r in range(2):
        for key, bad in ((25, float("nan")), (120 if r == 0 else 90, float("inf")), (159 if r == 0 else 110, float("-inf"))):
            b.cache[int(b.tables[r, key // 16]), :, :, key % 16] = bad
    got, _ = run(b, window=40, prefix=20)
    check(got, want)
    b.cache[int(b.tables[0, 12]), 1, 0, 0, 7] = float("nan")     # key 192 of the first request, which sees it
    got, _ = run(b, window=40, prefix=20)
    assert torch.isnan(got[0, :2, 7]).all() and torch.isfinite(got[0, 2:]).all() and torch.isfinite(got[1]).all()
    keep = torch.arange(128, device=DEV) != 7
    assert torch.isfinite(got[0, :2][:, keep]).all()
    b.q[1, 3, 0] = float("nan")
    got, _ = run(b, window=40, prefix=20)
    assert torch.isnan(got[1, 3]).all() and torch.isfinite(got[1, :3]).all()


def test_without_modifications_it_is_plain_decode():
    b = Batch(8, 2, 128, [300, 17, 1000], [1] * 3, seed=6)
    got, _ = run(b)
    assert torch.equal(got, b.pool.attn_decode(0, b.q, b.tables, b.seq_lens, b.scale))


def test_bad_block_ids_are_skipped_and_latched():
    b = Batch(4, 2, 64, [99], [1], seed=7)
    want, _ = run(b, window=20)
    b.tables[0, 1] = 1 << 20                                       # outside the window: never read
    got, _ = run(b, window=20)
    assert torch.equal(got, want) and b.pool.poll_status() == ekv.Status.OK
    b.tables[0, 6] = -1
    got = b.pool.attn_decode_scored(0, b.q, b.tables, b.seq_lens, b.scale, window=20)
    torch.cuda.synchronize()
    assert torch.isfinite(got).all() and b.pool.poll_status() == ekv.Status.ERR_BLOCK_OOB


def test_replayed_while_the_sequences_grow():
    b = Batch(8, 2, 64, [700, 90], [1, 1], seed=8, stale=False)
    slopes, out = slopes_of(8), torch.empty_like(b.q)
    lens = b.seq_lens.clone()
    ws = b.pool.workspace(2, b.tables.shape[1] * 16)
    call = lambda: b.pool.attn_decode_scored(0, b.q, b.tables, lens, b.scale, cap=9.0, window=200, slopes=slopes, out=out, workspace=ws)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for n in ([701, 91], [650, 1], [300, 80]):
        lens.copy_(torch.tensor(n, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        b.lens, b.past = n, [x - 1 for x in n]
        check(out, b.model(cap=9.0, window=200, slopes=slopes))


def test_refusals():
    b = Batch(4, 2, 64, [99], [1], seed=9)
    call = lambda **k: b.pool.attn_decode_scored(0, b.q, b.tables, b.seq_lens, k.pop("scale", b.scale), **k)
    for bad in ({"cap": -1.0}, {"cap": float("nan")}, {"cap": float("inf")}, {"window": -1}, {"scale": float("nan")}):
        with pytest.raises(ekv.EkvError) as e:
            call(**bad)
        assert e.value.status == ekv.Status.ERR_INVALID, bad
    for bad in ({"slopes": slopes_of(4).double()}, {"slopes": slopes_of(5)}, {"prefix_lens": torch.zeros(2, dtype=torch.int32, device=DEV)},
                {"prefix_lens": torch.zeros(1, dtype=torch.int32)}, {"out": torch.empty_like(b.q[:, :2])}):
        with pytest.raises(ValueError):
            call(**bad)
    e4m3 = ekv.Pool(num_q_heads=4, num_kv_heads=2, head_dim=64, base_blocks=16, dtype=ekv.EKV_E4M3)
    with pytest.raises(ekv.EkvError):
        e4m3.attn_decode_scored(0, b.q, b.tables, b.seq_lens, b.scale, cap=3.0)
    long = torch.zeros((1, 4000), dtype=torch.int32, device=DEV)
    with pytest.raises(ekv.EkvError) as e:
        b.pool.attn_decode_scored(0, b.q, long, b.seq_lens, b.scale, workspace=torch.empty(256, dtype=torch.uint8, device=DEV))
    assert e.value.status == ekv.Status.ERR_WORKSPACE
    assert b.pool.attn_decode_scored(0, b.q[:0], b.tables[:0], b.seq_lens[:0], b.scale, cap=1.0).shape == (0, 4, 64)


def test_workspaces_belong_to_the_streams_that_use_them():
    b, side = Batch(8, 2, 128, [5011, 800], [1, 1], seed=12), torch.cuda.Stream()
    want = b.pool.attn_decode_scored(0, b.q, b.tables, b.seq_lens, b.scale, cap=9.0)
    out = torch.empty_like(want)
    torch.cuda.synchronize()
    b.pool.attn_decode_scored(0, b.q, b.tables, b.seq_lens, b.scale, cap=9.0, out=out, stream=side)
    side.synchronize()
    assert torch.equal(out, want)
    mine = b.pool._parts[side.cuda_stream][-1].data_ptr()
    assert [s["stream"] for s in torch.cuda.memory_snapshot() if s["address"] <= mine < s["address"] + s["total_size"]] == [side.cuda_stream]
    graph = torch.cuda.CUDAGraph()      # captured on a stream, the call given another one that was forked from it
    out.zero_()
    with torch.cuda.graph(graph):
        main = torch.cuda.current_stream()
        side.wait_stream(main)
        b.pool.attn_decode_scored(0, b.q, b.tables, b.seq_lens, b.scale, cap=9.0, out=out, stream=side)
        main.wait_stream(side)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)


@pytest.mark.parametrize("Hq,Hk,D", [(8, 2, 128), (5, 1, 64), (8, 8, 64), (16, 2, 128)])
def test_ranges_of_a_sequence_in_one_launch(Hq, Hk, D):
    lens = [2048, 1793, 257, 256, 1, 2000, 513]                     # up to eight ranges, some sequences fewer than the table has room for
    b = Batch(Hq, Hk, D, [x - 1 for x in lens], [1] * len(lens), seed=Hq)
    b.seq_lens[3] = b.lens[3] = 0
    got, want = run(b, window=1900, cap=20.0)
    check(got, want)
    assert (got[3] == 0).all()
    b.cache[int(b.tables[0, 600 // 16]), 0, 0, 600 % 16, 5] = float("nan")      # key 600 of the first, kv-head 0: the third of its ranges
    hurt = run(b, window=1900, cap=20.0)[0]
    assert torch.isnan(hurt[0, :Hq // Hk]).all()
    hurt[0, :Hq // Hk] = got[0, :Hq // Hk]
    assert torch.equal(hurt, got)
    short = b.seq_lens.clone()
    b.seq_lens[0] = b.lens[0] = 500                                 # the key lies behind the end
    check(*run(b, cap=20.0))
    b.seq_lens.copy_(short)
