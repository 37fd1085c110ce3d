"""Prefill attention with capped, biased and windowed scores and visible prefixes against the model in 64 bits."""
import pytest
import torch

import paper_2608_23658_b200 as ekv
from scored_model import BF16, DEV, Batch, check, slopes_of

pytestmark = pytest.mark.gpu
LAYOUTS = [(4, 2, 64), (28, 4, 128), (8, 8, 64), (6, 2, 128), (5, 1, 64), (64, 8, 128)]
MODS = [{}, {"cap": 30.0}, {"window": 37}, {"bias": True}, {"prefix": 200}, {"cap": 5.0, "window": 150, "bias": True, "prefix": 18}, {"window": 1},
        {"window": 128, "prefix": 128}, {"cap": 50.0, "bias": True}, {"bias": True, "prefix": 150}, {"cap": 8.0, "window": 20}]


def run(b, cap=0.0, window=0, bias=False, prefix=0, scale=None, skip=(), **more):
    n = len(b.lens)
    slopes = slopes_of(b.Hq) if bias else None
    pre = [prefix] * n if isinstance(prefix, int) else prefix
    use = torch.tensor(pre, dtype=torch.int32, device=DEV) if any(pre) else None
    got = b.pool.attn_prefill_chunk_scored(0, b.q, b.tables, b.cu, b.cu_host, b.seq_lens, b.scale if scale is None else scale, cap=cap, window=window,
                                           slopes=slopes, prefix_lens=use, **more)
    return got, b.model(scale=scale, cap=cap, window=window, slopes=slopes, prefix=pre if use is not None else None, skip=skip)


@pytest.mark.parametrize("mods", MODS, ids=str)
@pytest.mark.parametrize("Hq,Hk,D", LAYOUTS)
def test_against_the_model(Hq, Hk, D, mods):
    past, new = [0, 0, 100, 16, 0, 250, 0, 3], [1, 130, 5, 33, 0, 129, 300, 128]
    b = Batch(Hq, Hk, D, past, new, seed=Hq + D, magnitude=4.0 if "cap" in mods else 1.0)
    got, want = run(b, **mods)
    check(got, want, str(mods))
    assert b.pool.poll_status() == ekv.Status.OK


@pytest.mark.parametrize("mods", [{}, {"cap": 20.0}, {"window": 4000, "prefix": 50}, {"bias": True, "window": 9000}], ids=str)
@pytest.mark.parametrize("past,new", [([20011], [1]), ([9000], [40]), ([15, 7000], [3, 64]), ([30000], [7])], ids=str)
def test_few_rows_over_many_keys(past, new, mods):
    b = Batch(8, 2, 128, past, new, seed=5, magnitude=3.0, table_extra=40)
    got, want = run(b, **mods)
    check(got, want, str(mods))


@pytest.mark.parametrize("R", [256, 257, 700])
def test_many_requests(R):
    new = [(7 * r) % 23 for r in range(R)]
    b = Batch(4, 2, 64, [(5 * r) % 40 for r in range(R)], new, seed=R)
    got, want = run(b, window=30, cap=9.0)
    check(got, want)


def test_a_call_of_more_items_than_the_machine_holds():
    b = Batch(32, 8, 128, [0, 513, 0], [1500, 700, 129], seed=11)
    got, want = run(b, cap=30.0)
    check(got, want)
    for _ in range(3):
        assert torch.equal(run(b, cap=30.0)[0], got)


def test_prefixes_of_every_length_and_scales_of_any_sign():
    b = Batch(4, 2, 64, [0, 20, 0, 10, 0], [90, 90, 90, 90, 300], seed=2)
    check(*run(b, window=10, prefix=[5, -3, 90, 2000, 131]))
    for scale in (-0.2, 0.0):
        for cap in (0.0, 4.0):
            check(*run(b, cap=cap, scale=scale, window=50), f"scale {scale} cap {cap}")


def test_scores_far_beyond_the_cap():
    b = Batch(4, 2, 64, [200, 0], [40, 160], seed=3, magnitude=500.0)
    for cap in (1.0, 50.0):
        check(*run(b, cap=cap))


def test_caps_of_any_size_and_queries_of_zeros():
    b = Batch(4, 2, 64, [200, 0], [40, 160], seed=16, magnitude=20.0)
    for cap in (1e-42, 1e-30, 1e-3, 3e3, 1e6, 1e30):
        check(*run(b, cap=cap), str(cap))
    b.q.zero_()
    for cap in (1e-42, 1e-30, 50.0, 1e6):
        check(*run(b, cap=cap), str(cap))


def test_malformed_requests_come_out_as_zeros():
    b = Batch(8, 2, 128, [10, 10, 3000], [200, 30, 5], seed=12)
    for lens in ([210, 29, 3005], [210, 40, 4]):
        b.seq_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        bad = [r for r in range(3) if lens[r] < b.new[r]]
        got, (want, bound) = run(b, window=100, skip=bad)
        torch.cuda.synchronize()
        assert b.pool.poll_status() == (ekv.Status.ERR_BLOCK_OOB)
        for r in range(3):
            rows = slice(int(b.cu_host[r]), int(b.cu_host[r + 1]))
            if r in bad:
                assert (got[rows] == 0).all()
            elif lens[r] == b.lens[r]:
                check(got[rows], (want[rows], bound[rows]))
    one = Batch(8, 2, 128, [3000], [5], seed=13)                    # its keys would be cut into parts
    one.seq_lens[0] = 4
    assert (run(one, skip=[0])[0] == 0).all()


@pytest.mark.parametrize("past,new", [([100], [90]), ([2000], [4]), ([0], [200])], ids=str)
def test_what_a_row_does_not_see_does_not_reach_it(past, new):
    b = Batch(8, 2, 128, past, new, seed=4)
    n, c, window = past[0] + new[0], new[0], 64
    got, (want, bound) = run(b, window=window)
    check(got, (want, bound))
    V = lambda key: b.cache[int(b.tables[0, key // 16]), 1, :, key % 16]
    bad = {n - 1: (3, float("nan")), max(n - c - window + 2, 0): (5, float("inf")), n - c // 2 - 1: (9, float("-inf")), n - c // 2: (9, float("inf"))}
    for key, (ch, v) in bad.items():
        V(key)[:, ch] = v
    got = run(b, window=window, skip=[0])[0]
    for i in range(c):
        p = n - c + i
        for ch in range(128):
            seen = [v for key, (k, v) in bad.items() if k == ch and p - window < key <= p]
            if not seen:
                continue
            x = sum(seen)
            col = got[i, :, ch].float()
            assert torch.isnan(col).all() if x != x else (col == x).all(), (i, ch, seen)
            got[i, :, ch] = want[i, :, ch].to(BF16)
    assert torch.isfinite(got).all()
    check(got, (want, bound * 1.01))                                # (what was put in is rounded once more)


def test_a_bad_key_or_query_reaches_the_rows_that_see_it():
    b = Batch(4, 2, 64, [0], [300], seed=14)
    want = run(b, window=50)[0]
    b.cache[int(b.tables[0, 6]), 0, 0, 4, 10] = float("nan")        # key 100, kv-head 0
    b.q[250, 3, 1] = float("nan")
    got = run(b, window=50, skip=[0])[0]
    hit = torch.zeros(300, 4, dtype=torch.bool, device=DEV)
    hit[100:150, :2], hit[250, 3] = True, True
    assert torch.isnan(got[hit]).all() and torch.equal(got[~hit], want[~hit])


def test_bad_block_ids_are_skipped_and_latched():
    b = Batch(4, 2, 64, [500], [20], seed=7)
    want, _ = run(b, window=40)
    b.tables[0, 3] = 1 << 20                                        # outside every window: never read
    got, _ = run(b, window=40, skip=[0])
    torch.cuda.synchronize()
    assert torch.equal(got, want) and b.pool.poll_status() == ekv.Status.OK
    b.tables[0, 31] = -1
    got, _ = run(b, window=40, skip=[0])
    torch.cuda.synchronize()
    assert torch.isfinite(got).all() and b.pool.poll_status() == ekv.Status.ERR_BLOCK_OOB


def test_without_modifications_it_is_plain_prefill_within_rounding():
    b = Batch(32, 8, 128, [500, 0], [200, 77], seed=15)
    got, (want, bound) = run(b)
    plain = b.pool.attn_prefill_chunk(0, b.q, b.tables, b.cu, b.cu_host, b.seq_lens, b.scale)
    assert ((got.double() - plain.double()).abs() <= 2 * bound).all()


def test_replayed_side_by_side():
    b = Batch(8, 2, 64, [700, 90], [30, 200], seed=8)
    slopes = slopes_of(8)
    want = b.model(cap=9.0, window=200, slopes=slopes)
    run(b, cap=9.0, window=200, bias=True)
    graphs, outs, kept, streams = [], [], [], [torch.cuda.Stream(), torch.cuda.Stream()]
    need = ekv.ekv_attn_prefill_scored_workspace_bytes(b.pool.handle)
    torch.cuda.synchronize()
    for _ in range(2):
        g, out, ws = torch.cuda.CUDAGraph(), torch.zeros_like(b.q), torch.empty(need, dtype=torch.uint8, device=DEV)
        with torch.cuda.graph(g):
            b.pool.attn_prefill_chunk_scored(0, b.q, b.tables, b.cu, b.cu_host, b.seq_lens, b.scale, cap=9.0, window=200, slopes=slopes, out=out, workspace=ws)
        graphs.append(g), outs.append(out), kept.append(ws)             # (a graph does not keep what it was handed)
    for _ in range(5):
        for s, g in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for out in outs:
        check(out, want)


def test_refusals():
    b = Batch(4, 2, 64, [2000], [3], seed=9)
    def call(q=b.q, cu=b.cu, cu_host=b.cu_host, scale=b.scale, **k):
        return b.pool.attn_prefill_chunk_scored(0, q, b.tables, cu, cu_host, b.seq_lens, scale, **k)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32)
    for bad in ({"cap": -1.0}, {"cap": float("nan")}, {"window": -1}, {"scale": float("inf")}, {"cu_host": i32(1, 3)}):
        with pytest.raises(ekv.EkvError) as e:
            call(**bad)
        assert e.value.status == ekv.Status.ERR_INVALID, bad
    for bad in ({"slopes": slopes_of(8)}, {"prefix_lens": torch.zeros(2, dtype=torch.int32, device=DEV)}, {"q": b.q[:2]}, {"q": b.q.float()},
                {"cu_host": i32(0, 1, 3)}, {"cu_host": b.cu}, {"cu": b.cu_host}, {"out": torch.empty_like(b.q[:2])}):
        with pytest.raises(ValueError):
            call(**bad)
    with pytest.raises(ekv.EkvError) as e:
        call(workspace=torch.empty(256, dtype=torch.uint8, device=DEV))
    assert e.value.status == ekv.Status.ERR_WORKSPACE
    e4m3 = ekv.Pool(num_q_heads=4, num_kv_heads=2, head_dim=64, base_blocks=16, dtype=ekv.EKV_E4M3)
    with pytest.raises(ekv.EkvError):
        e4m3.attn_prefill_chunk_scored(0, b.q, b.tables, b.cu, b.cu_host, b.seq_lens, b.scale, cap=3.0)


# A few more items than SMs, over long tables.
SECOND_ROUND = [
    (32, 8, 128, [9000], [1300], 0, {"cap": 30.0}),                    # 168 items
    (28, 4, 128, [8500], [1400], 0, {"bias": True}),                   # 156, whose rows end inside a position's heads
    (5, 1, 64, [700], [8000], 0, {"prefix": 8400}),
    (8, 8, 64, [4000], [4900], 0, {"window": 8300}),                   # 160, a head each
    (32, 8, 128, [9000, 3, 0, 100], [1100, 40, 0, 200], 0, {}),
    (32, 8, 128, [100, 3, 0, 9000], [200, 40, 0, 1100], 0, {}),
    (32, 8, 128, [0], [1300], 700, {"cap": 30.0}),                     # long tables, few keys
    (32, 8, 128, [0, 1200], [700, 700], 700, {}),
]


@pytest.mark.parametrize("Hq,Hk,D,past,new,extra,mods", SECOND_ROUND, ids=str)
def test_a_second_round_of_items(Hq, Hk, D, past, new, extra, mods):
    b = Batch(Hq, Hk, D, past, new, seed=Hq + D, table_extra=extra, magnitude=4.0 if "cap" in mods else 1.0)
    got, want = run(b, **mods)
    check(got, want, str(mods))
    for _ in range(3):
        assert torch.equal(run(b, skip=range(len(new)), **mods)[0], got)


def test_a_second_round_with_values_that_are_not_finite_and_a_malformed_request():
    b = Batch(32, 8, 128, [9000, 5000], [700, 600], seed=21)
    got, (want, bound) = run(b)
    check(got, (want, bound))
    key = 5000 + 300                                                # of the second request, seen by its rows from 300 on
    b.cache[int(b.tables[1, key // 16]), 1, :, key % 16, 7] = float("inf")
    key = 9000 + 20                                                 # of the first
    b.cache[int(b.tables[0, key // 16]), 1, 2, key % 16, 9] = float("nan")
    hurt = run(b, skip=[0, 1])[0]
    assert (hurt[1000:, :, 7] == float("inf")).all() and torch.isnan(hurt[20:700, 8:12, 9]).all()
    hurt[1000:, :, 7], hurt[20:700, 8:12, 9] = got[1000:, :, 7], got[20:700, 8:12, 9]
    assert torch.equal(hurt, got)
    b.seq_lens[0] = 699
    hurt = run(b, skip=[0, 1])[0]
    torch.cuda.synchronize()
    assert (hurt[:700] == 0).all() and b.pool.poll_status() == ekv.Status.ERR_BLOCK_OOB
