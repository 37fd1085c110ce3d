"""8-bit pools on the GPU: write, read, decode and prefill against the 64-bit models of e4m3_model.py."""
import math

import numpy as np
import pytest
import torch

import e4m3_model as M
import ekv_inputs as I
import paper_2608_23658_b200 as ekv

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
SHAPES = [I.TINY, I.LLAMA8B, I.LLAMA70B, I.Shape(28, 4, 128), I.Shape(8, 8, 64), I.Shape(5, 1, 64), I.Shape(6, 2, 128)]


def make_pool(shape, base_blocks, **kw):
    return ekv.Pool(num_q_heads=shape.num_q_heads, num_kv_heads=shape.num_kv_heads, head_dim=shape.head_dim,
                    base_blocks=base_blocks, dtype=ekv.EKV_E4M3, **kw)


def rows(rng, T, shape, spread=3.0):
    """bf16 rows whose heads and tokens differ in magnitude, so that scales differ and rise."""
    x = rng.standard_normal((T, shape.num_kv_heads, shape.head_dim)) * 2.0 ** rng.uniform(-spread, spread, (T, shape.num_kv_heads, 1))
    return torch.from_numpy(x).to(torch.bfloat16)


def same_bits(pool, cache, layer=0):
    """The pool's codes and scales of a layer are the model's, NaN codes of either sign being one."""
    n = len(cache.codes)
    codes = pool.layer_tensor(layer, 0, n).contiguous().view(torch.uint8).cpu().numpy()
    scales = pool.layer_scales(layer, 0, n).cpu().numpy().astype(np.float64)
    codes = np.where(codes == 0xFF, 0x7F, codes)
    want = np.where(cache.codes == 0xFF, 0x7F, cache.codes)
    assert np.array_equal(scales, cache.scales), np.argwhere(scales != cache.scales)[:5]
    assert np.array_equal(codes, want), np.argwhere(codes != want)[:5]


def fresh(shape, blocks, **kw):
    pool = make_pool(shape, blocks, **kw)
    live = pool.info.live_blocks
    for layer in range(pool.num_layers):
        pool.layer_tensor(layer).view(torch.uint8).fill_(0x7F)  # NaN wherever nothing is written
    return pool, M.Cache(live, shape.num_kv_heads, shape.head_dim)


def write_both(pool, cache, k, v, slots, layer=0):
    slots = torch.as_tensor(np.asarray(slots), dtype=torch.int64)
    pool.write_kv(layer, k.to(DEV), v.to(DEV), slots.to(DEV))
    return cache.write(k.double().numpy(), v.double().numpy(), slots.numpy())


# ------------------------------------------------------------------------------------------ write and read


@pytest.mark.parametrize("shape", [I.TINY, I.LLAMA8B, I.Shape(5, 1, 64)], ids=str)
@pytest.mark.parametrize("T", [1, 2, 16, 17, 333, 1024, 1025, 1500])
def test_write_orders(shape, T):
    """Runs, scattered and shuffled slots, in one call and in several, on both sides of the length where the launch changes."""
    rng = np.random.default_rng(T)
    pool, cache = fresh(shape, 200)
    with pool:
        live = len(cache.codes)
        run = (np.arange(T) + 5) % (live * 16)
        k, v = rows(rng, T, shape), rows(rng, T, shape)
        assert not write_both(pool, cache, k, v, run)
        same_bits(pool, cache)
        mixed = rng.permutation(live * 16)[:T]
        assert not write_both(pool, cache, rows(rng, T, shape), rows(rng, T, shape), mixed)
        same_bits(pool, cache)
        some = np.where(rng.random(T) < 0.3, -1, rng.permutation(live * 16)[:T])
        write_both(pool, cache, rows(rng, T, shape), rows(rng, T, shape), some)
        same_bits(pool, cache)
        assert pool.poll_status() == ekv.Status.OK
        back = rng.integers(0, live * 16, 50)
        kk, vv = pool.read_kv(0, torch.from_numpy(back).to(DEV))
        wk, wv = cache.rows(back)
        assert np.array_equal(kk.double().cpu().numpy(), wk, equal_nan=True) and np.array_equal(vv.double().cpu().numpy(), wv, equal_nan=True)


def test_write_token_by_token_is_like_the_model():
    shape, rng = I.TINY, np.random.default_rng(3)
    pool, cache = fresh(shape, 8)
    with pool:
        for pos in range(40):  # one sequence over three blocks, a token a call, its magnitude growing and falling
            k, v = rows(rng, 1, shape, 8), rows(rng, 1, shape, 8)
            write_both(pool, cache, k, v, [[3, 1, 6][pos // 16] * 16 + pos % 16])
        same_bits(pool, cache)
        write_both(pool, cache, rows(rng, 1, shape, 0), rows(rng, 1, shape, 0), [3 * 16])  # the block passes to another request
        same_bits(pool, cache)


@pytest.mark.parametrize("T", [300, 2000])
def test_write_duplicate_slots_and_out_of_range(T):
    """Of duplicate slots the last wins, alone: neither the others' values nor their magnitudes stay."""
    shape, rng = I.TINY, np.random.default_rng(T)
    pool, cache = fresh(shape, 256)
    with pool:
        live = len(cache.codes)
        slots = rng.integers(0, 40 * 16, T)
        slots[::7] = -1
        slots[5::31] = live * 16 + rng.integers(0, 1 << 40, len(slots[5::31]))
        assert write_both(pool, cache, rows(rng, T, shape, 6), rows(rng, T, shape, 6), slots)
        same_bits(pool, cache)
        assert pool.poll_status() == ekv.Status.ERR_BLOCK_OOB and pool.poll_status() == ekv.Status.OK


def test_write_values_at_the_edges():
    shape, rng = I.TINY, np.random.default_rng(9)
    pool, cache = fresh(shape, 16)
    with pool:
        big = float(torch.finfo(torch.bfloat16).max)
        for n, put in enumerate([[0.0], [-0.0, 1e-40, -1e-40], [2.0 ** -112 * 448, 2.0 ** -120], [448.0, 447.0], [450.0, -450.0], [big, -big, 1.0],
                                 [np.nan, 3.0], [np.inf, -np.inf, 5.0], [np.nan], [-np.inf, big], [1.0, 2.0 ** -10, 2.0 ** -17]]):
            x = rng.standard_normal((20, 2, 64)) if n > 9 else np.zeros((20, 2, 64))
            x[:, :, :len(put)] = put
            k = torch.from_numpy(x).to(torch.bfloat16)
            write_both(pool, cache, k[:9], k[11:], np.arange(9) + 16 * n)
            write_both(pool, cache, k[9:11] * 4, k[9:11], np.array([9, 12]) + 16 * n)  # beside the ones that are there
            same_bits(pool, cache)
        k, v = pool.read_kv(0, torch.arange(5 * 16, 6 * 16).to(DEV))
        assert torch.isfinite(k[:9]).all() and float(k[0, 0, 0]) == 240 * 2.0 ** 120


def test_read_kv_of_a_bf16_pool_and_untouched_rows():
    shape, rng = I.LLAMA8B, np.random.default_rng(5)
    for dtype in (ekv.EKV_BF16, ekv.EKV_E4M3):
        with ekv.Pool(num_q_heads=32, num_kv_heads=8, head_dim=128, base_blocks=64, dtype=dtype) as pool:
            k, v = rows(rng, 100, shape).to(DEV), rows(rng, 100, shape).to(DEV)
            slots = torch.from_numpy(rng.permutation(64 * 16)[:100]).to(DEV)
            pool.write_kv(0, k, v, slots)
            ask = slots.clone()
            ask[3], ask[50], ask[99] = -1, 10 ** 9, slots[0]
            ko, vo = torch.full_like(k, 7.0), torch.full_like(v, 7.0)
            pool.read_kv(0, ask, ko, vo)
            torch.cuda.synchronize()
            assert pool.poll_status() == ekv.Status.ERR_BLOCK_OOB
            assert (ko[[3, 50]] == 7).all() and (vo[[3, 50]] == 7).all()
            assert torch.equal(ko[99], ko[0]) and torch.equal(vo[99], vo[0])
            keep = torch.ones(100, dtype=torch.bool, device=DEV)
            keep[[3, 50, 99]] = False
            if dtype == ekv.EKV_BF16:
                assert torch.equal(ko[keep], k[keep]) and torch.equal(vo[keep], v[keep])
            else:
                # scattered tokens may share a block: half a code's step of the block's largest element at most
                assert ((ko[keep].double() - k[keep].double()).abs() <= k.double().abs().max() * 2.0 ** -4).all()
            e = torch.empty(0, dtype=torch.int64, device=DEV)
            pool.read_kv(0, e)
            pool.write_kv(0, k[:0], v[:0], e)


@pytest.mark.parametrize("fused", [False, True])
def test_layers_elastic_blocks_and_moves(fused):
    """Blocks of every layer keep codes and scales through grow, move_blocks and shrink; both halves of the range are written."""
    shape, rng = I.TINY, np.random.default_rng(11)
    pool, _ = fresh(shape, 512, elastic_blocks=512, num_layers=3, fused_range=fused, start_grown=True)
    with pool:
        info = pool.info
        base, live = info.base_blocks, info.live_blocks
        caches = [M.Cache(live, 2, 64) for _ in range(3)]
        for layer in range(3):
            slots = rng.permutation(live * 16)[:1200]
            write_both(pool, caches[layer], rows(rng, 1200, shape), rows(rng, 1200, shape), slots, layer)
        for layer in range(3):
            same_bits(pool, caches[layer], layer)
        src, dst = np.arange(base, base + 40), np.arange(100, 140)
        pool_move = torch.from_numpy(np.stack([src, dst]).astype(np.int32)).to(DEV)
        ekv.ekv_move_blocks(pool.handle, pool_move[0].contiguous(), pool_move[1].contiguous())
        for c in caches:
            c.codes[dst], c.scales[dst] = c.codes[src], c.scales[src]
        for layer in range(3):
            same_bits(pool, caches[layer], layer)
        pool.shrink()
        k = rows(rng, 4, shape)
        pool.write_kv(0, k.to(DEV), k.to(DEV), torch.tensor([base * 16, 1, 2, 3], device=DEV))
        torch.cuda.synchronize()
        assert pool.poll_status() == ekv.Status.ERR_BLOCK_OOB
        caches[0].write(k[1:].double().numpy(), k[1:].double().numpy(), [1, 2, 3])
        for c in caches:
            c.codes, c.scales = c.codes[:base], c.scales[:base]
        for layer in range(3):
            same_bits(pool, caches[layer], layer)
        pool.grow()
        assert pool.poll_status() == ekv.Status.OK


@pytest.mark.parametrize("dtype", [ekv.EKV_BF16, ekv.EKV_E4M3])
@pytest.mark.parametrize("k_at,v_at", [(8, 0), (0, 8), (8, 8)])  # elements: 16 bytes past a 32-byte boundary
def test_read_kv_into_outputs_on_16_byte_boundaries(dtype, k_at, v_at):
    rng = np.random.default_rng(6)
    with ekv.Pool(num_q_heads=4, num_kv_heads=2, head_dim=64, base_blocks=64, dtype=dtype) as pool:
        n = 37 * 2 * 64
        pool.write_kv(0, rows(rng, 37, I.TINY).to(DEV), rows(rng, 37, I.TINY).to(DEV), torch.arange(37).to(DEV))
        at = torch.from_numpy(rng.permutation(37)).to(DEV)
        want = pool.read_kv(0, at)
        flat = [torch.full((n + 32,), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
        got = [f[s:s + n].view(37, 2, 64) for f, s in zip(flat, (k_at, v_at))]
        pool.read_kv(0, at, *got)
        for f, s, g, w in zip(flat, (k_at, v_at), got, want):
            assert torch.equal(g, w) and (f[:s] == 7).all() and (f[s + n:] == 7).all()



def test_write_on_streams_and_in_a_replayed_graph():
    shape, rng = I.TINY, np.random.default_rng(12)
    pool, cache = fresh(shape, 400, num_layers=2)
    other = M.Cache(len(cache.codes), 2, 64)
    with pool:
        T = 3000
        a, b = rows(rng, T, shape), rows(rng, T, shape)
        slots = torch.from_numpy(rng.permutation(400 * 16)[:T])
        half = slots // 16 % 2 == 0  # two calls at once: the same layer with blocks of its own each, and another layer
        s1, s2, s3 = (torch.cuda.Stream() for _ in range(3))
        da, db, ds, d1, d2 = a.to(DEV), b.to(DEV), slots.to(DEV), torch.where(half, slots, -1).to(DEV), torch.where(half, -1, slots).to(DEV)
        torch.cuda.synchronize()
        pool.write_kv(0, da, db, d1, stream=s1)
        pool.write_kv(0, da, db, d2, stream=s2)
        pool.write_kv(1, db, da, ds, stream=s3)
        torch.cuda.synchronize()
        cache.write(a.double().numpy(), b.double().numpy(), slots.numpy())
        other.write(b.double().numpy(), a.double().numpy(), slots.numpy())
        same_bits(pool, cache, 0)
        same_bits(pool, other, 1)
        for n in (200, T):  # both launches
            k, v, at = da[:n].clone(), db[:n].clone(), ds[:n].clone()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                pool.write_kv(0, k, v, at)
            for _ in range(3):
                nk, nv, ns = rows(rng, n, shape, 5), rows(rng, n, shape, 5), rng.permutation(400 * 16)[:n]
                k.copy_(nk), v.copy_(nv), at.copy_(torch.from_numpy(ns))
                g.replay()
                cache.write(nk.double().numpy(), nv.double().numpy(), ns)
                same_bits(pool, cache)


# ------------------------------------------------------------------------------------------ attention


class Case:
    """Sequences quantised into a pool; K and V are the stored values (float64) of each."""

    def __init__(self, shape, lengths, seed, id_lo=0, **kw):
        rng = np.random.default_rng(seed)
        self.shape, self.lengths = shape, [int(x) for x in lengths]
        need = sum(-(-L // 16) for L in self.lengths)
        self.pool = make_pool(shape, need + 3, **kw)
        live = self.pool.info.live_blocks
        self.pool.layer_tensor(0).view(torch.uint8).fill_(0x7F)
        self.tables, _ = I.assign_blocks(seed, 4, torch.tensor(self.lengths), 16, live - id_lo, id_lo=id_lo)
        if self.tables.shape[1] == 0:
            self.tables = torch.full((len(self.lengths), 1), -1, dtype=torch.int32)
        self.slots = [I.position_slots(self.tables[b], 0, L, 16) if L else torch.empty(0, dtype=torch.int64) for b, L in enumerate(self.lengths)]
        slots = torch.cat(self.slots)
        k, v = rows(rng, len(slots), shape, 1.5), rows(rng, len(slots), shape, 1.5)
        for i in range(0, len(slots), 5000):
            self.pool.write_kv(0, k[i:i + 5000].to(DEV), v[i:i + 5000].to(DEV), slots[i:i + 5000].to(DEV))
        # values as stored: the write and the read have tests of their own
        kk, vv = self.pool.read_kv(0, slots.to(DEV))
        kk, vv, at = kk.double().cpu(), vv.double().cpu(), 0
        self.K, self.V = [], []
        for L in self.lengths:
            self.K.append(kk[at:at + L])
            self.V.append(vv[at:at + L])
            at += L
        self.V_ids = [s // 16 for s in self.slots]
        self.d_tables = self.tables.to(torch.int32).to(DEV)
        self.d_lens = torch.tensor(self.lengths, dtype=torch.int32, device=DEV)
        self.rng = rng

    def sv(self, b, L=None):
        """V's scale of every key of a sequence, as the pool has it now."""
        return self.pool.layer_scales(0)[self.V_ids[b][:L].to(DEV), 1].double().cpu()

    def queries(self, n, mag=1.0):
        s = self.shape
        return torch.from_numpy(self.rng.standard_normal((n, s.num_q_heads, s.head_dim)) * mag).to(torch.bfloat16)

    def check_decode(self, q, out, scale, what=""):
        for b, L in enumerate(self.lengths):
            want, bound = M.attention(q[b:b + 1].double(), self.K[b], self.V[b], [L], scale, self.sv(b))
            M.assert_within(out[b:b + 1], want, bound, f"{what} sequence {b} of {L}")


@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_decode_lengths(shape):
    c = Case(shape, [0, 1, 15, 16, 17, 63, 64, 65, 255, 256, 257, 1000, 2049], seed=21)
    with c.pool:
        q, scale = c.queries(len(c.lengths)), 1 / math.sqrt(shape.head_dim)
        out = c.pool.attn_decode(0, q.to(DEV), c.d_tables, c.d_lens, scale)
        c.check_decode(q, out, scale)
        again = c.pool.attn_decode(0, q.to(DEV), c.d_tables, c.d_lens, scale)
        static = torch.empty_like(out)
        ekv.ekv_attn_decode_static_scratch(c.pool.handle, 0, q.to(DEV), static, c.d_tables, c.d_lens, scale)
        assert torch.equal(out, again) and torch.equal(out, static)
        assert c.pool.poll_status() == ekv.Status.OK


@pytest.mark.parametrize("shape", [I.TINY, I.LLAMA8B], ids=str)
def test_decode_one_and_many(shape):
    """One long sequence (many key ranges), a batch so large that a sequence is one range, and a single key."""
    for lengths in ([9001], [33] * 700, [1]):
        c = Case(shape, lengths, seed=len(lengths))
        with c.pool:
            q, scale = c.queries(len(lengths)), 1 / math.sqrt(shape.head_dim)
            out = c.pool.attn_decode(0, q.to(DEV), c.d_tables, c.d_lens, scale)
            if len(lengths) > 100:
                c.lengths = c.lengths[:40]
            c.check_decode(q, out, scale)


def test_decode_magnitudes_and_scales():
    """Queries of any magnitude and either sign of the scale; keys and values whose blocks' scales lie far apart."""
    shape = I.LLAMA8B
    c = Case(shape, [700, 40], seed=31)
    with c.pool:
        for mag, scale in ((1e-30, 0.1), (1e30, 1e-30), (300.0, 1e-3), (1.0, -0.1), (1.0, 0.0)):
            q = c.queries(2, mag)
            out = c.pool.attn_decode(0, q.to(DEV), c.d_tables, c.d_lens, scale)
            c.check_decode(q, out, scale, f"queries x {mag}, scale {scale}")
        # every block's K and V scale moved by a power of two of its own: V's by up to 2^40
        n = c.pool.info.live_blocks
        sc = c.pool.layer_scales(0, 0, n)
        up = torch.from_numpy(c.rng.integers(-20, 21, (n, 2, 8))).to(DEV).float()
        up[:, 0] = up[:, 0].clamp(-3, 1)
        sc *= torch.exp2(up)
        slots = torch.cat(c.slots)
        kk, vv = c.pool.read_kv(0, slots.to(DEV))
        c.K, c.V = [kk[:700].double().cpu(), kk[700:].double().cpu()], [vv[:700].double().cpu(), vv[700:].double().cpu()]
        q = c.queries(2)
        out = c.pool.attn_decode(0, q.to(DEV), c.d_tables, c.d_lens, 0.05)
        c.check_decode(q, out, 0.05, "scales far apart")


def test_decode_skips_invalid_blocks():
    shape = I.TINY
    c = Case(shape, [200, 100, 16], seed=41)
    with c.pool:
        t = c.d_tables.clone()
        t[0, 3], t[0, 7], t[1, 0], t[2, 0] = -1, 1 << 30, -5, 1 << 20
        for b, j in ((0, 3), (0, 7), (1, 0), (2, 0)):
            c.K[b][16 * j:16 * j + 16] = float("nan")
        q = c.queries(3)
        out = c.pool.attn_decode(0, q.to(DEV), t, c.d_lens, 0.125)
        c.check_decode(q, out, 0.125)
        assert (out[2] == 0).all()
        assert c.pool.poll_status() == ekv.Status.ERR_BLOCK_OOB


def test_decode_over_long_offsets_on_a_stream_in_a_graph():
    """A block id whose byte offset passes 32 bits; the call captured on a side stream and replayed with other lengths."""
    shape = I.LLAMA8B
    blocks = (5 << 30) // (32 * 1024)
    c = Case(shape, [500, 37], seed=51, id_lo=blocks, elastic_blocks=blocks + 64, start_grown=True)
    with c.pool:
        assert int(c.tables.max()) * 32 * 1024 > 1 << 32
        q = c.queries(2).to(DEV)
        out, ws = torch.empty_like(q), c.pool.workspace(2, c.d_tables.shape[1] * 16).clone()
        side = torch.cuda.Stream()
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g, stream=side):
            c.pool.attn_decode(0, q, c.d_tables, c.d_lens, 0.09, out=out, workspace=ws)
        for lens in ([500, 37], [1, 0], [499, 16]):
            c.d_lens.copy_(torch.tensor(lens, dtype=torch.int32))
            q.copy_(c.queries(2))
            g.replay()
            for b, L in enumerate(lens):
                want, bound = M.attention(q[b:b + 1].double().cpu(), c.K[b][:L], c.V[b][:L], [L], 0.09, c.sv(b, L))
                M.assert_within(out[b:b + 1], want, bound)


def test_hoststep_runs_on_an_8_bit_pool():
    shape = I.LLAMA8B
    c = Case(shape, [100, 33, 16], seed=61)
    with c.pool:
        step = ekv.HostStep(c.pool, 4, c.tables.shape[1])
        q, k, v = c.queries(3).pin_memory(), rows(c.rng, 3, shape).pin_memory(), rows(c.rng, 3, shape).pin_memory()
        slots = torch.stack([s[-1] for s in c.slots]).pin_memory()
        out = torch.empty_like(q).pin_memory()
        step.decode(0, q, c.tables.to(torch.int32).contiguous().pin_memory(), torch.tensor(c.lengths, dtype=torch.int32).pin_memory(), 0.1, out, k, v, slots)
        step.flush()
        torch.cuda.synchronize()
        after = [c.pool.read_kv(0, s.to(DEV)) for s in c.slots]
        c.K, c.V = [a[0].double().cpu() for a in after], [a[1].double().cpu() for a in after]
        c.check_decode(q, out, 0.1)
        step.close()


def check_prefill(c, chunks, scale=None, mag=1.0, tables=None, what=""):
    """Request r's last chunks[r] tokens as its query rows."""
    scale = 1 / math.sqrt(c.shape.head_dim) if scale is None else scale
    cu = torch.tensor(np.concatenate([[0], np.cumsum(chunks)]), dtype=torch.int32)
    q = c.queries(int(cu[-1]), mag)
    out = torch.full_like(q, 7.0).to(DEV)
    c.pool.attn_prefill_chunk(0, q.to(DEV), c.d_tables if tables is None else tables, cu.to(DEV), cu, c.d_lens, scale, out=out)
    for r, (n, L) in enumerate(zip(chunks, c.lengths)):
        a, b = int(cu[r]), int(cu[r + 1])
        if n > L:
            assert (out[a:b] == 0).all(), what
        elif n:
            want, bound = M.attention(q[a:b].double(), c.K[r], c.V[r], torch.arange(L - n, L) + 1, scale, c.sv(r))
            M.assert_within(out[a:b], want, bound, f"{what} request {r}: {n} rows of {L}")
    return q, cu, out


@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_prefill_shapes(shape):
    """Whole prompts, chunks over prefixes, single rows and empty requests; lengths around tiles of keys, items of rows and blocks."""
    lengths = [1, 2, 16, 17, 0, 127, 128, 129, 300, 513, 40, 260, 255, 700]
    chunks = [1, 1, 16, 17, 0, 127, 128, 129, 300, 200, 1, 256, 5, 33]
    c = Case(shape, lengths, seed=71)
    with c.pool:
        q, cu, out = check_prefill(c, chunks)
        again = c.pool.attn_prefill_chunk(0, q.to(DEV), c.d_tables, cu.to(DEV), cu, c.d_lens, 1 / math.sqrt(shape.head_dim))
        assert torch.equal(out, again)
        assert c.pool.poll_status() == ekv.Status.OK


@pytest.mark.parametrize("shape", [I.TINY, I.LLAMA8B, I.Shape(28, 4, 128)], ids=str)
def test_prefill_long_and_many(shape):
    c = Case(shape, [3000], seed=81)
    with c.pool:
        for n in (3000, 1, 65, 777):
            check_prefill(c, [n])
    rng = np.random.default_rng(8)
    lengths = rng.integers(1, 60, 300)  # more requests than the launch parameters hold offsets for
    c = Case(shape, lengths, seed=82)
    with c.pool:
        check_prefill(c, [int(rng.integers(0, L + 1)) for L in lengths])
        assert c.pool.poll_status() == ekv.Status.OK


@pytest.mark.parametrize("shape", [I.TINY, I.LLAMA8B, I.Shape(5, 1, 64)], ids=str)
def test_prefill_few_rows_over_long_and_wide_tables(shape):
    """Few rows (both slots on the same ones), keys cut over clusters of every size, and tables so much wider than the
    sequences that some of a cluster's CTAs have no keys."""
    for lengths, chunks, width in (([5000], [3], 0), ([2600, 1, 900], [4, 1, 130], 0), ([130, 5, 300, 256], [40, 5, 2, 256], 700),
                                   ([700] * 40, [5] * 40, 0), ([1500] * 9, [100] * 9, 300)):
        c = Case(shape, lengths, seed=sum(lengths))
        with c.pool:
            if width:
                wide = torch.full((len(lengths), width), 1 << 30, dtype=torch.int32, device=DEV)
                wide[:, :c.d_tables.shape[1]] = c.d_tables
                c.d_tables = wide
            _, cu, out = check_prefill(c, chunks, what=f"{lengths[:4]}, {chunks[:4]}")
            assert c.pool.poll_status() == ekv.Status.OK


def test_prefill_magnitudes_and_scales():
    shape = I.Shape(6, 2, 128)
    c = Case(shape, [400, 40], seed=83)
    with c.pool:
        for mag, scale in ((1e-30, 0.1), (1e30, 1e-30), (300.0, 1e-3), (1.0, -0.1), (1.0, 0.0), (1e-38, 1e-3)):
            check_prefill(c, [150, 40], scale, mag, what=f"queries x {mag}, scale {scale}")
        n = c.pool.info.live_blocks
        up = torch.from_numpy(c.rng.integers(-20, 21, (n, 2, 2))).to(DEV).float()
        up[:, 0] = up[:, 0].clamp(-3, 1)
        c.pool.layer_scales(0, 0, n).mul_(torch.exp2(up))
        kk, vv = c.pool.read_kv(0, torch.cat(c.slots).to(DEV))
        c.K, c.V = [kk[:400].double().cpu(), kk[400:].double().cpu()], [vv[:400].double().cpu(), vv[400:].double().cpu()]
        check_prefill(c, [150, 40], 0.05, what="scales far apart")


def test_prefill_invalid_blocks_and_requests():
    shape = I.LLAMA8B
    c = Case(shape, [300, 40, 16, 500, 3, 77], seed=84)
    with c.pool:
        t = c.d_tables.clone()
        for b, j, bad in ((0, 3, -1), (0, 17, 1 << 30), (2, 0, -9), (3, 0, 1 << 20)):
            t[b, j] = bad
            c.K[b][16 * j:16 * j + 16] = float("nan")
        q, cu, out = check_prefill(c, [300, 41, 16, 129, 9, 60], tables=t)  # the second and fifth have fewer keys than rows
        assert (out[int(cu[2]):int(cu[3])] == 0).all()  # a request whose every key is skipped
        assert c.pool.poll_status() == ekv.Status.ERR_BLOCK_OOB


def test_never_written_blocks_read_as_zero():
    """Scale 0: the values are 0, whatever the codes (here NaN); and V blocks of zeros, whose scale is the smallest there is."""
    shape = I.TINY
    c = Case(shape, [64, 100], seed=85)
    with c.pool:
        ids = c.tables[0, 1:3].long()
        c.pool.layer_scales(0)[ids.to(DEV)] = 0.0
        c.pool.layer_tensor(0).view(torch.uint8)[ids.to(DEV)] = 0x7F
        c.K[0][16:48], c.V[0][16:48] = 0.0, 0.0
        for x in c.pool.read_kv(0, c.slots[0][16:48].to(DEV)):
            assert (x == 0).all()
        # many keys whose values are 0 and whose scores are not the lowest: their weights count
        zero = torch.zeros(80, 2, 64, dtype=torch.bfloat16)
        k = rows(c.rng, 80, shape, 1.0)
        c.pool.write_kv(0, k.to(DEV), zero.to(DEV), c.slots[1][:80].to(DEV))
        kk, vv = c.pool.read_kv(0, c.slots[1].to(DEV))
        c.K[1], c.V[1] = kk.double().cpu(), vv.double().cpu()
        assert float(c.pool.layer_scales(0)[int(c.tables[1, 0]), 1].max()) == 2.0 ** -112
        for chunks in ([64, 100], [3, 2], [20, 9], [0, 40]):
            check_prefill(c, chunks)
        q = c.queries(2)
        c.check_decode(q, c.pool.attn_decode(0, q.to(DEV), c.d_tables, c.d_lens, 0.125), 0.125)


def test_prefill_on_streams_and_in_a_replayed_graph():
    shape = I.LLAMA8B
    c = Case(shape, [700, 333, 90], seed=86)
    with c.pool:
        cu = torch.tensor([0, 200, 533, 560], dtype=torch.int32)
        qs = [c.queries(560).to(DEV) for _ in range(4)]
        dcu, want = cu.to(DEV), []
        for q in qs:
            want.append(c.pool.attn_prefill_chunk(0, q, c.d_tables, dcu, cu, c.d_lens, 0.09))
        torch.cuda.synchronize()
        streams, got = [torch.cuda.Stream() for _ in qs], [torch.empty_like(q) for q in qs]
        for s, q, o in zip(streams, qs, got):
            c.pool.attn_prefill_chunk(0, q, c.d_tables, dcu, cu, c.d_lens, 0.09, out=o, stream=s)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got))
        q, o = qs[0].clone(), torch.empty_like(qs[0])
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c.pool.attn_prefill_chunk(0, q, c.d_tables, dcu, cu, c.d_lens, 0.09, out=o)
        for a, b in zip(qs, want):
            q.copy_(a)
            g.replay()
            assert torch.equal(o, b)


def test_captured_prefills_replayed_side_by_side():
    """Two captured calls of more items than the GPU has SMs, captured any number of calls apart, share no state."""
    shape = I.LLAMA8B
    c = Case(shape, [257, 300, 280, 266] * 3, seed=88)
    with c.pool:
        cu = torch.tensor([0, *np.cumsum([257, 200, 280, 66] * 3)], dtype=torch.int32)
        dcu, n = cu.to(DEV), int(cu[-1])
        qs = [c.queries(n).to(DEV) for _ in range(2)]
        want = [c.pool.attn_prefill_chunk(0, q, c.d_tables, dcu, cu, c.d_lens, 0.09) for q in qs]
        outs, graphs, streams = [torch.empty_like(q) for q in qs], [], [torch.cuda.Stream() for _ in qs]
        few = torch.tensor([0, 16] + [16] * 11, dtype=torch.int32)
        d_few = few.to(DEV)
        for q, o in zip(qs, outs):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                c.pool.attn_prefill_chunk(0, q, c.d_tables, dcu, cu, c.d_lens, 0.09, out=o)
            graphs.append(g)
            for _ in range(63):
                c.pool.attn_prefill_chunk(0, q[:16], c.d_tables, d_few, few, c.d_lens, 0.09)
        for _ in range(20):
            for o in outs:
                o.zero_()
            torch.cuda.synchronize()
            for g, s in zip(graphs, streams):
                with torch.cuda.stream(s):
                    g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(want, outs))
        assert c.pool.poll_status() == ekv.Status.OK


def test_mixed_call_is_through_before_what_follows():
    """A long chunk and a single row are two launches side by side: the next operation on the stream finds both results."""
    shape = I.LLAMA8B
    c = Case(shape, [3000, 20], seed=90)
    with c.pool:
        cu = torch.tensor([0, 1500, 1501], dtype=torch.int32)
        q, dcu = c.queries(1501).to(DEV), cu.to(DEV)
        want = c.pool.attn_prefill_chunk(0, q, c.d_tables, dcu, cu, c.d_lens, 0.09)
        torch.cuda.synchronize()
        out = torch.empty_like(want)
        for _ in range(10):
            out.fill_(7.0)
            c.pool.attn_prefill_chunk(0, q, c.d_tables, dcu, cu, c.d_lens, 0.09, out=out)
            assert torch.equal(out.clone(), want)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out.fill_(7.0)
            c.pool.attn_prefill_chunk(0, q, c.d_tables, dcu, cu, c.d_lens, 0.09, out=out)
            copy = out.clone()
        for _ in range(10):
            g.replay()
            assert torch.equal(copy, want)
        assert c.pool.poll_status() == ekv.Status.OK


def test_prompt_in_chunks_then_decode_steps():
    """A run as it would be used: chunks written and attended to one after the other, then single tokens; every result against the
    cache's own values, and the last decode step against the prefill of that one row."""
    shape, rng = I.LLAMA8B, np.random.default_rng(87)
    pool, _ = fresh(shape, 64)
    with pool:
        free, cursor = torch.from_numpy(rng.permutation(64).astype(np.int32)).to(DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
        lens, tables = torch.zeros(1, dtype=torch.int32, device=DEV), torch.full((1, 40), -1, dtype=torch.int32, device=DEV)
        for n in (100, 37, 250, 1, 1, 130, 1, 1):
            slots, cu = torch.zeros(n, dtype=torch.int64, device=DEV), torch.zeros(2, dtype=torch.int32, device=DEV)
            pool.extend_tables(torch.tensor([n], dtype=torch.int32, device=DEV), lens, tables, free, cursor, slots, cu)
            k, v = rows(rng, n, shape, 1.5).to(DEV), rows(rng, n, shape, 1.5).to(DEV)
            pool.write_kv(0, k, v, slots)
            q = torch.from_numpy(rng.standard_normal((n, 32, 128))).to(torch.bfloat16)
            L = int(lens)
            at = tables[0, torch.arange(L, device=DEV) // 16].long() * 16 + torch.arange(L, device=DEV) % 16
            kk, vv = (x.double().cpu() for x in pool.read_kv(0, at))
            want, bound = M.attention(q.double(), kk, vv, torch.arange(L - n, L) + 1, 0.09, pool.layer_scales(0)[at // 16, 1].double().cpu())
            out = pool.attn_prefill_chunk(0, q.to(DEV), tables, cu, torch.tensor([0, n], dtype=torch.int32), lens, 0.09)
            M.assert_within(out, want, bound, f"{n} rows of {L}")
            if n == 1:
                M.assert_within(pool.attn_decode(0, q.to(DEV), tables, lens, 0.09), want, bound, f"token {L}")
        assert pool.poll_status() == ekv.Status.OK


def test_a_view_keeps_its_pool():
    """The pool goes with its last name or view, whichever is later."""
    import weakref
    pool = make_pool(I.TINY, 64)
    ref = weakref.ref(pool)
    codes, scales = pool.layer_tensor(0, 0, 3)[1:], pool.layer_scales(0, 0, 3).view(-1)
    del pool
    assert ref() is not None
    del codes
    assert ref() is not None and ref().handle
    scales.fill_(2.0)
    assert float(scales.sum()) == 2.0 * 3 * 2 * 2
    del scales
    assert ref() is None


def test_refusals():
    shape = I.TINY
    with make_pool(shape, 64) as pool:
        q = torch.zeros(1, 4, 64, dtype=torch.bfloat16, device=DEV)
        t, n = torch.zeros(1, 1, dtype=torch.int32, device=DEV), torch.ones(1, dtype=torch.int32, device=DEV)
        second = torch.zeros(pool.info.block_bytes, dtype=torch.uint8, device=DEV)
        with pytest.raises(ekv.EkvError) as e:
            ekv.ekv_attn_decode_two_tensor(pool.handle, 0, second, q, torch.empty_like(q), t, n, 1.0, pool.workspace(1, 16))
        assert e.value.status == ekv.Status.ERR_INVALID
        with pytest.raises(ekv.EkvError) as e:
            ekv.ekv_attn_decode(pool.handle, 0, q, torch.empty_like(q), t, n, 1.0, None)
        assert e.value.status == ekv.Status.ERR_WORKSPACE
        lib, s = ekv.load_library(), torch.zeros(4, dtype=torch.int64, device=DEV)
        for k_out, v_out, slots, T in ((None, q.data_ptr(), s.data_ptr(), 1), (q.data_ptr() + 2, q.data_ptr(), s.data_ptr(), 1),
                                       (q.data_ptr(), q.data_ptr(), None, 1), (q.data_ptr(), q.data_ptr(), s.data_ptr(), -1)):
            assert lib.ekv_read_kv(pool.handle, 0, k_out, v_out, slots, T, None) == ekv.Status.ERR_INVALID
        assert lib.ekv_read_kv(pool.handle, 1, q.data_ptr(), q.data_ptr(), s.data_ptr(), 1, None) == ekv.Status.ERR_INVALID
        assert pool.poll_status() == ekv.Status.OK
