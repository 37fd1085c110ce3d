"""Decode attention of batches whose requests share prefixes against the model in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2608_23658_b200 as ekv
from scored_model import BF16, DEV, Batch, check

pytestmark = pytest.mark.gpu


def make(Hq, Hk, D, groups, own, seed=0, **more):
    """groups: (requests, shared tokens); own: own tokens of each request (repeated as needed)."""
    past, share, starts = [], [], [0]
    for n, p in groups:
        first = len(past)
        for i in range(n):
            past.append(p + own[len(past) % len(own)] - 1)
            share.append((first, p // 16 if i else 0))
        starts.append(len(past))
    b = Batch(Hq, Hk, D, past, [1] * len(past), seed=seed, share=share, **more)
    b.starts = torch.tensor(starts, dtype=torch.int32)
    b.shared = torch.tensor([p for _, p in groups], dtype=torch.int32)
    return b


def run(b, **more):
    return b.pool.attn_decode_shared(0, b.q, b.tables, b.seq_lens, b.starts, b.shared, b.scale, **more)


@pytest.mark.parametrize("Hq,Hk,D", [(4, 2, 64), (28, 4, 128), (8, 8, 64), (6, 2, 128), (5, 1, 64), (64, 8, 128)])
@pytest.mark.parametrize("groups,own", [
    ([(1, 64)], [5]), ([(2, 16)], [1, 40]), ([(4, 512)], [1, 17, 40, 16]), ([(3, 128), (1, 256), (5, 0), (2, 2000)], [3, 100, 15]),
    ([(40, 304)], [1, 9, 33]), ([(70, 1040), (0, 0), (33, 48)], [20, 64])], ids=str)
def test_against_the_model(Hq, Hk, D, groups, own):
    b = make(Hq, Hk, D, groups, own, seed=len(own))
    check(run(b), b.model())
    assert b.pool.poll_status() == ekv.Status.OK


@pytest.mark.parametrize("Hq,Hk,D", [(4, 2, 64), (28, 4, 128), (8, 8, 64), (6, 2, 128), (5, 1, 64), (64, 8, 128)])
@pytest.mark.parametrize("groups,own", [
    ([(2, 12000)], [1, 40]), ([(2, 16), (4, 64), (2, 12000), (3, 128), (1, 48), (0, 0), (5, 0)], [3, 100, 15, 1]), ([(40, 11904), (3, 2000)], [1, 9, 33]),
    ([(37, 1040), (70, 12016), (33, 48)], [20, 64]), ([(2, 36000)], [1, 40]), ([(2, 16), (4, 64), (2, 36000), (3, 128), (1, 48), (0, 0), (5, 0)], [3, 100, 15, 1])], ids=str)
def test_beside_a_prefix_that_is_long_enough_to_be_read_once(Hq, Hk, D, groups, own):
    b = make(Hq, Hk, D, groups, own, seed=len(own))
    assert ekv.ekv_attn_decode_shared_workspace_bytes(b.pool.handle, b.starts, b.shared, b.tables.shape[1]) > 0
    check(run(b), b.model())
    assert b.pool.poll_status() == ekv.Status.OK


@pytest.mark.parametrize("Hq,Hk,D,n,p,own", [(32, 8, 128, 256, 4096, [1, 50]), (8, 1, 128, 3, 40000, [7]), (4, 2, 64, 130, 10000, [300]),
                                              (8, 2, 128, 2, 1024, [5000, 9000])])
def test_large_groups_and_long_prefixes(Hq, Hk, D, n, p, own):
    b = make(Hq, Hk, D, [(n, p)], own, seed=n)
    check(run(b), b.model())


@pytest.mark.parametrize("p", [160, 12000, 36000])
def test_requests_that_have_no_keys_of_their_own(p):
    b = make(8, 2, 128, [(5, p), (2, 32)], [16], seed=1)
    b.seq_lens[1], b.seq_lens[4], b.seq_lens[6] = p, p, 32
    b.lens[1], b.lens[4], b.lens[6] = p, p, 32
    check(run(b), b.model())


@pytest.mark.parametrize("p", [320, 12000, 36000])
def test_rows_of_padding_and_requests_shorter_than_their_prefix(p):
    b = make(4, 2, 64, [(6, p), (3, 0)], [30], seed=2)
    want = run(b)
    assert b.pool.poll_status() == ekv.Status.OK
    b.seq_lens[2], b.seq_lens[7] = 0, 0
    got = run(b)
    torch.cuda.synchronize()
    keep = [r for r in range(9) if r not in (2, 7)]
    assert (got[[2, 7]] == 0).all() and torch.equal(got[keep], want[keep]) and b.pool.poll_status() == ekv.Status.OK
    b.seq_lens[4] = p - 1
    got = run(b)
    torch.cuda.synchronize()
    assert (got[4] == 0).all() and b.pool.poll_status() == ekv.Status.ERR_BLOCK_OOB
    keep.remove(4)
    assert torch.equal(got[keep], want[keep])


def test_as_plain_decode_within_rounding_and_the_same_bits_every_time():
    b = make(28, 4, 128, [(9, 12000), (1, 480), (4, 96)], [100, 3, 700], seed=3)
    got, plain = run(b), b.pool.attn_decode(0, b.q, b.tables, b.seq_lens, b.scale)
    want, bound = b.model()
    assert ((got.double() - plain.double()).abs() <= 2 * bound).all()
    for _ in range(4):
        assert torch.equal(run(b), got)


@pytest.mark.parametrize("p", [256, 12000, 36000])
def test_a_nan_reaches_its_own_request_alone(p):
    b = make(8, 2, 64, [(6, p)], [20], seed=4)
    want = run(b)
    b.cache[int(b.tables[3, p // 16]), 1, 1, 2, 9] = float("nan")      # an own value of request 3
    b.q[5, 0, 0] = float("nan")
    got = run(b)
    assert torch.isnan(got[3, 4:, 9]).all() and torch.isnan(got[5, 0]).all()
    got[3, 4:, 9], want[3, 4:, 9] = 0, 0
    got[5, 0], want[5, 0] = 0, 0
    assert torch.equal(got, want)
    b.cache[int(b.tables[0, 3]), 0, 0, 0, 0] = float("nan")       # a shared key of kv-head 0: all its rows
    assert torch.isnan(run(b)[:, :4]).all() and torch.isfinite(run(b)[[0, 1, 2, 4]][:, 4:]).all()


@pytest.mark.parametrize("p", [400, 12000, 36000])
def test_bad_shared_block_ids_are_skipped_and_latched(p):
    b = make(8, 2, 128, [(4, p)], [20], seed=5)
    want = run(b)
    b.tables[1:, :p // 16] = 1 << 24                                     # only the first request's are read
    assert torch.equal(run(b), want) and b.pool.poll_status() == ekv.Status.OK
    b.tables[0, 7] = -5
    got = run(b)
    torch.cuda.synchronize()
    assert torch.isfinite(got).all() and b.pool.poll_status() == ekv.Status.ERR_BLOCK_OOB


def test_replayed_while_the_requests_grow_two_graphs_side_by_side():
    b = make(8, 2, 128, [(20, 8000), (3, 64)], [70, 200], seed=6, stale=False)
    need = ekv.ekv_attn_decode_shared_workspace_bytes(b.pool.handle, b.starts, b.shared, b.tables.shape[1])
    lens, outs, graphs, kept = b.seq_lens.clone(), [], [], []
    run(b)
    torch.cuda.synchronize()
    for _ in range(2):
        ws, out = torch.empty(need, dtype=torch.uint8, device=DEV), torch.empty_like(b.q)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            b.pool.attn_decode_shared(0, b.q, b.tables, lens, b.starts, b.shared, b.scale, out=out, workspace=ws)
        outs.append(out), graphs.append(g), kept.append(ws)             # (a graph does not keep what it was handed)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for drop in (0, 13, 60):
        lens.copy_(b.seq_lens - drop)
        torch.cuda.synchronize()
        for _ in range(3):
            for s, g in zip(streams, graphs):
                with torch.cuda.stream(s):
                    g.replay()
        torch.cuda.synchronize()
        full = b.lens
        b.lens = [x - drop for x in full]
        model = b.model()
        b.lens = full
        for out in outs:
            check(out, model)


def test_refusals():
    b = make(4, 2, 64, [(3, 64), (2, 32)], [10], seed=7)
    call = lambda starts=b.starts, shared=b.shared, scale=b.scale, **k: b.pool.attn_decode_shared(0, b.q, b.tables, b.seq_lens, starts, shared, scale, **k)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32)
    for bad in ({"starts": i32(0, 3, 4)}, {"starts": i32(1, 3, 5)}, {"starts": i32(0, 6, 5)}, {"shared": i32(64, 33)}, {"shared": i32(-16, 32)},
                {"shared": i32(64, 1 << 20)}, {"scale": 0.0}, {"scale": -1.0}, {"scale": float("nan")},
                {"starts": torch.arange(258, dtype=torch.int32).clamp(max=5), "shared": torch.zeros(257, dtype=torch.int32)}):
        with pytest.raises(ekv.EkvError) as e:
            call(**bad)
        assert e.value.status == ekv.Status.ERR_INVALID, bad
    for bad in ({"starts": b.starts.long()}, {"starts": i32(0, 5)}, {"shared": b.shared.to(DEV)}, {"out": torch.empty_like(b.q).float()}):
        with pytest.raises(ValueError):
            call(**bad)
    long = make(4, 2, 64, [(3, 12000)], [10], seed=7)
    with pytest.raises(ekv.EkvError) as e:
        run(long, workspace=torch.empty(256, dtype=torch.uint8, device=DEV))
    assert e.value.status == ekv.Status.ERR_WORKSPACE
    e4m3 = ekv.Pool(num_q_heads=4, num_kv_heads=2, head_dim=64, base_blocks=16, dtype=ekv.EKV_E4M3)
    with pytest.raises(ekv.EkvError):
        e4m3.attn_decode_shared(0, b.q, b.tables, b.seq_lens, b.starts, b.shared, b.scale)
    none = b.pool.attn_decode_shared(0, b.q[:0], b.tables[:0], b.seq_lens[:0], i32(0), i32(), b.scale)
    assert none.shape == (0, 4, 64)
