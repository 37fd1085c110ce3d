"""ekv_extend_tables against a plain loop, its refusals, and whole steps made of it."""
import math

import numpy as np
import pytest
import torch

import e4m3_model as M
import paper_2608_23658_b200 as ekv

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def model(new, lens, tables, free, cursor, T_cap):
    """(tables, lens, cursor, slots, cu) after the step."""
    tables, slots, cu = tables.copy(), np.full(T_cap, -1, np.int64), [0]
    for r, (n, l) in enumerate(zip(new, lens)):
        for i in range(int(n)):
            p = int(l) + i
            if p % 16 == 0:
                tables[r, p // 16] = free[cursor]
                cursor += 1
            slots[cu[-1] + i] = int(tables[r, p // 16]) * 16 + p % 16
        cu.append(cu[-1] + int(n))
    return tables, np.asarray(lens) + np.asarray(new), cursor, slots, np.array(cu)


def dev(a, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV).to(dtype)


@pytest.fixture(scope="module")
def pool():
    with ekv.Pool(num_q_heads=2, num_kv_heads=1, head_dim=64, base_blocks=1 << 17, dtype=ekv.EKV_E4M3) as p:
        yield p


class Step:
    def __init__(self, rng, R, hi, past, spare, width_spare=2, T_spare=3):
        self.new = rng.integers(0, hi + 1, R)
        self.lens = rng.integers(0, past + 1, R)
        have = -(-self.lens // 16)
        self.width = max(1, int((-(-(self.lens + self.new) // 16)).max(initial=0)) + width_spare)
        self.need = int((-(-(self.lens + self.new) // 16) - have).sum())
        ids = rng.permutation(1 << 17)[:int(have.sum()) + self.need + spare].astype(np.int32)
        self.tables = np.full((R, self.width), -7, np.int32)
        at = 0
        for r in range(R):
            self.tables[r, :have[r]] = ids[at:at + have[r]]
            at += have[r]
        self.free = np.concatenate([np.full(5, -9, np.int32), ids[at:]])  # five ids already taken
        self.T_cap = int(self.new.sum()) + T_spare

    def put(self):
        self.d = dict(new_tokens=dev(self.new), seq_lens=dev(self.lens), block_tables=dev(self.tables), free_ids=dev(self.free),
                      free_cursor=dev([5]), slot_mapping=torch.full((self.T_cap,), 99, dtype=torch.int64, device=DEV),
                      cu_q_lens=torch.full((len(self.new) + 1,), 99, dtype=torch.int32, device=DEV))
        return self.d

    def check(self, d, lens, cursor):
        t, l, c, s, cu = model(self.new, self.lens, self.tables, self.free, 5, self.T_cap)
        for got, want in ((d["block_tables"], t), (lens, l), (cursor, [c]), (d["slot_mapping"], s), (d["cu_q_lens"], cu)):
            assert np.array_equal(got.cpu().numpy(), want)


@pytest.mark.parametrize("R,hi,past", [(1, 1, 0), (1, 1, 40), (1, 3000, 17), (3, 40, 100), (64, 1, 500), (257, 1, 300), (513, 33, 100),
                                       (1000, 100, 64), (16384, 2, 40), (7, 0, 50), (2, 20000, 5)])
def test_like_the_plain_loop(pool, R, hi, past):
    rng = np.random.default_rng(R * 1000 + hi)
    s = Step(rng, R, hi, past, spare=4)
    d = s.put()
    lens, cursor = torch.zeros_like(d["seq_lens"]), torch.zeros_like(d["free_cursor"])
    pool.extend_tables(**d, seq_lens_out=lens, free_cursor_out=cursor)
    s.check(d, lens, cursor)
    assert np.array_equal(d["seq_lens"].cpu().numpy(), s.lens) and int(d["free_cursor"]) == 5
    d = s.put()
    pool.extend_tables(**d)  # in place
    s.check(d, d["seq_lens"], d["free_cursor"])
    assert pool.poll_status() == ekv.Status.OK


def test_nothing_to_do(pool):
    e = torch.empty(0, dtype=torch.int32, device=DEV)
    slots, cu, cursor = torch.zeros(9, dtype=torch.int64, device=DEV), torch.full((1,), 5, dtype=torch.int32, device=DEV), dev([0])
    pool.extend_tables(e, e.clone(), torch.empty(0, 1, dtype=torch.int32, device=DEV), e.clone(), cursor, slots, cu)
    assert (slots == -1).all() and int(cu) == 0 and int(cursor) == 0
    one = dev([0])
    pool.extend_tables(one, dev([16]), torch.full((1, 1), 3, dtype=torch.int32, device=DEV), e, cursor, slots[:0], torch.zeros(2, dtype=torch.int32, device=DEV))
    assert pool.poll_status() == ekv.Status.OK


@pytest.mark.parametrize("big", [False, True])  # one CTA, and a cluster
@pytest.mark.parametrize("fault,status", [("short list", "ERR_OOM"), ("tokens", "ERR_INVALID"), ("row", "ERR_INVALID"), ("negative new", "ERR_INVALID"),
                                          ("negative length", "ERR_INVALID"), ("sum past 32 bits", "ERR_INVALID"), ("free id", "ERR_BLOCK_OOB"),
                                          ("free id negative", "ERR_BLOCK_OOB"), ("partial block", "ERR_BLOCK_OOB"), ("cursor", "ERR_OOM")])
def test_refused_whole(pool, big, fault, status):
    rng = np.random.default_rng(77)
    s = Step(rng, 300, 40 if big else 5, 90, spare=0)
    s.new[7], s.lens[7] = 3, 5  # a partly filled block
    s.T_cap = int(s.new.sum()) + 40
    cursor = 5
    have = -(-s.lens // 16)
    s.need = int((-(-(s.lens + s.new) // 16) - have).sum())
    s.free = np.concatenate([np.full(5, -9), np.arange(s.need)]).astype(np.int32)
    for r in range(300):
        s.tables[r, :have[r]] = 1000 + r
    if fault == "short list":
        s.free = s.free[:-1]
    elif fault == "tokens":
        s.T_cap = int(s.new.sum()) - 1
    elif fault == "row":
        s.lens[7] = s.width * 16 - 2
    elif fault == "negative new":
        s.new[7] = -1
    elif fault == "negative length":
        s.lens[7] = -1
    elif fault == "sum past 32 bits":
        s.new[7] = 2 ** 31 - 1
    elif fault == "free id":
        s.free[-1] = 1 << 17
    elif fault == "free id negative":
        s.free[5] = -1
    elif fault == "partial block":
        s.tables[7, 0] = 1 << 20
    elif fault == "cursor":
        cursor = -1
    d = s.put()
    d["free_cursor"].fill_(cursor)
    before = d["block_tables"].clone()
    lens, out = torch.full_like(d["seq_lens"], 55), torch.full_like(d["free_cursor"], 55)
    pool.extend_tables(**d, seq_lens_out=lens, free_cursor_out=out)
    assert torch.equal(d["block_tables"], before) and torch.equal(lens, d["seq_lens"]) and int(out) == cursor
    assert (d["slot_mapping"] == -1).all() and (d["cu_q_lens"] == 0).all()
    assert pool.poll_status() == getattr(ekv.Status, status) and pool.poll_status() == ekv.Status.OK


def test_refused_arguments(pool):
    rng = np.random.default_rng(1)
    d = Step(rng, 4, 3, 3, 1).put()
    lib, P = ekv.load_library(), {k: v.data_ptr() for k, v in d.items()}

    def call(**kw):
        a = dict(P, R=4, width=3, n_free=1, T_cap=1) | kw
        return lib.ekv_extend_tables(pool.handle, a["new_tokens"], a["seq_lens"], a["R"], a["block_tables"], a["width"], a["free_ids"], a["n_free"],
                                     a["free_cursor"], a["slot_mapping"], a["T_cap"], a["cu_q_lens"], a["seq_lens"], a["free_cursor"], None)

    for kw in (dict(R=-1), dict(R=16385), dict(width=0), dict(n_free=-1), dict(T_cap=-1), dict(T_cap=(1 << 30) + 1), dict(new_tokens=None),
               dict(seq_lens=None), dict(block_tables=None), dict(free_ids=None), dict(free_cursor=None), dict(slot_mapping=None), dict(cu_q_lens=None)):
        assert call(**kw) == ekv.Status.ERR_INVALID, kw
    torch.cuda.synchronize()
    assert pool.poll_status() == ekv.Status.OK


@pytest.mark.parametrize("dtype", [ekv.EKV_BF16, ekv.EKV_E4M3])
def test_decode_steps_in_one_replayed_graph(dtype):
    """A captured step -- tables, write, attention -- replayed while requests grow over block borders with no word from the host."""
    rng = np.random.default_rng(5)
    R, Hq, Hk, D, steps, width = 5, 8, 2, 64, 40, 8
    with ekv.Pool(num_q_heads=Hq, num_kv_heads=Hk, head_dim=D, base_blocks=256, dtype=dtype) as pool:
        pool.layer_tensor(0).view(torch.uint8).fill_(0x7F)
        bp = ekv.ekv_blockpool_create(pool.info.base_blocks, 0)
        lease = np.array(ekv.ekv_blockpool_alloc(bp, 40), np.int32)
        rng.shuffle(lease)
        new, lens, tables = dev(np.ones(R)), dev([0, 15, 16, 40, 3]), torch.full((R, width), -1, dtype=torch.int32, device=DEV)
        free, cursor = dev(lease), dev([0])
        pad = R + 2
        slots, cu = torch.zeros(pad, dtype=torch.int64, device=DEV), torch.zeros(R + 1, dtype=torch.int32, device=DEV)
        # the tokens that the requests start with
        start = lens.clone()
        first_slots, first_cu = torch.zeros(int(start.sum()), dtype=torch.int64, device=DEV), torch.zeros(R + 1, dtype=torch.int32, device=DEV)
        lens.zero_()
        pool.extend_tables(start, lens, tables, free, cursor, first_slots, first_cu)
        history_k = [[] for _ in range(R)]
        history_v = [[] for _ in range(R)]
        k0, v0 = (torch.from_numpy(rng.standard_normal((int(start.sum()), Hk, D))).to(torch.bfloat16) for _ in range(2))
        pool.write_kv(0, k0.to(DEV), v0.to(DEV), first_slots)
        for r in range(R):
            a, b = int(first_cu[r]), int(first_cu[r + 1])
            history_k[r] += list(k0[a:b])
            history_v[r] += list(v0[a:b])
        q, k, v = (torch.zeros(pad, h, D, dtype=torch.bfloat16, device=DEV) for h in (Hq, Hk, Hk))
        out, ws = torch.zeros(R, Hq, D, dtype=torch.bfloat16, device=DEV), pool.workspace(R, width * 16).clone()
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            pool.extend_tables(new, lens, tables, free, cursor, slots, cu)
            pool.write_kv(0, k, v, slots)
            pool.attn_decode(0, q[:R], tables, lens, 1 / math.sqrt(D), out=out, workspace=ws)
        for step in range(steps):
            hq, hk, hv = (torch.from_numpy(rng.standard_normal((pad, h, D))).to(torch.bfloat16) for h in (Hq, Hk, Hk))
            q.copy_(hq), k.copy_(hk), v.copy_(hv)
            g.replay()
            for r in range(R):
                history_k[r].append(hk[r])
                history_v[r].append(hv[r])
            if step % 13 == 0 or step == steps - 1:
                for r in range(R):
                    L = int(lens[r])
                    assert L == len(history_k[r])
                    at = torch.from_numpy(model([L], [0], np.full((1, width), -1), tables[r].cpu().numpy(), 0, L)[3]).to(DEV)
                    kk, vv = pool.read_kv(0, at)
                    hist = torch.stack(history_k[r]).double()
                    step_of = hist.abs().max() * 2.0 ** -4 if dtype == ekv.EKV_E4M3 else 0.0
                    assert ((kk.double().cpu() - hist).abs() <= step_of).all()
                    sv = pool.layer_scales(0)[at // 16, 1].double().cpu() if dtype == ekv.EKV_E4M3 else None
                    want, bound = M.attention(hq[r:r + 1].double(), kk.double().cpu(), vv.double().cpu(), [L], 1 / math.sqrt(D), sv)
                    M.assert_within(out[r:r + 1], want, bound, f"step {step} request {r}")
        assert int(cursor) == sum(-(-len(h) // 16) for h in history_k)
        assert pool.poll_status() == ekv.Status.OK
        ekv.ekv_blockpool_destroy(bp)
