"""Attention over caches with NaN or infinite elements in valid slots: what sees one is NaN, everything else is as it would be."""
import math

import numpy as np
import pytest
import torch

import e4m3_model as M
import ekv_inputs as I
import paper_2608_23658_b200 as ekv
from test_gpu_e4m3 import DEV, rows

pytestmark = pytest.mark.gpu
DTYPES = [ekv.EKV_E4M3, ekv.EKV_BF16]


class Cache:
    """One sequence of L tokens in a pool of either type; `spoil` puts single elements into K or V on their way to write_kv.
    K, V: the stored values, float64; NaN where an element is not finite."""

    def __init__(self, dtype, shape, L, seed, spoil=()):
        self.rng, self.shape, self.L = np.random.default_rng(seed), shape, L
        blocks = -(-L // 16)
        self.pool = ekv.Pool(num_q_heads=shape.num_q_heads, num_kv_heads=shape.num_kv_heads, head_dim=shape.head_dim, base_blocks=blocks + 3, dtype=dtype)
        if dtype == ekv.EKV_E4M3:
            self.pool.layer_tensor(0).view(torch.uint8).fill_(0x7F)
        else:
            self.pool.layer_tensor(0).view(torch.int16).fill_(0x7FC0)
        ids = torch.from_numpy(self.rng.permutation(self.pool.info.live_blocks)[:blocks].astype(np.int32))
        self.tables = ids[None].to(DEV).contiguous()
        pos = torch.arange(L)
        slots = (ids[pos // 16].long() * 16 + pos % 16).to(DEV)
        kv = [rows(self.rng, L, shape, 1.5) for _ in range(2)]
        for which, t, h, x, value in spoil:
            kv["KV".index(which)][t, h, x] = value
        self.pool.write_kv(0, kv[0].to(DEV), kv[1].to(DEV), slots)
        self.K, self.V = (torch.where(torch.isfinite(y), y, math.nan) for y in (z.double().cpu() for z in self.pool.read_kv(0, slots)))
        self.lens = torch.tensor([L], dtype=torch.int32, device=DEV)
        self.sv = self.pool.layer_scales(0)[slots // 16, 1].double().cpu() if dtype == ekv.EKV_E4M3 else None

    def queries(self, n):
        return torch.from_numpy(self.rng.standard_normal((n, self.shape.num_q_heads, self.shape.head_dim))).to(torch.bfloat16)

    def want(self, q, limits, scale):
        """(out, bound): out is NaN where the row's head sees a NaN key or has one in the query, and in the channels of V that are
        NaN at a key that it sees."""
        limits = torch.as_tensor(limits)
        out, bound = M.attention(q.double().nan_to_num(0.0), self.K.nan_to_num(0.0), self.V.nan_to_num(0.0), limits, scale, self.sv)
        G = self.shape.num_q_heads // self.shape.num_kv_heads
        seen = torch.arange(self.L) < limits[:, None]                                     # [rows, L]
        key = (torch.isnan(self.K).any(2).double().T[:, None] * seen.double()).sum(2) > 0   # [Hk, rows]
        value = torch.einsum("rl,lhd->rhd", seen.double(), torch.isnan(self.V).double()) > 0
        nan = key.T.repeat_interleave(G, 1)[..., None] | value.repeat_interleave(G, 1) | torch.isnan(q).any(2, keepdim=True)
        return torch.where(nan, math.nan, out), bound


def check(got, want, bound, what=""):
    got = got.detach().cpu().double()
    nan = torch.isnan(want)
    assert torch.equal(torch.isnan(got), nan), f"{what}: {int((torch.isnan(got) & ~nan).sum())} NaN too many, {int((nan & ~torch.isnan(got)).sum())} too few"
    M.assert_within(torch.where(nan, 0.0, got), torch.where(nan, 0.0, want), bound, what)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", [I.TINY, I.LLAMA8B, I.Shape(28, 4, 128)], ids=str)
@pytest.mark.parametrize("L", [1, 40, 2500])
@pytest.mark.parametrize("value", [math.nan, math.inf])
def test_a_key_that_is_not_finite_reaches_every_kernel(dtype, shape, L, value):
    """One key of kv-head 1, so that other heads show what a tile beside it does; decode with one key range and with several,
    its combine pass and its static scratch, a prefill of one row, of some and of many."""
    if dtype == ekv.EKV_BF16 and value == math.inf:
        value = math.nan  # (an infinite bf16 key gives an infinite score, whose weight is 1 or 0 by its sign)
    c = Cache(dtype, shape, L, 7 + L, [("K", L // 2, 1, 5, value)])
    with c.pool:
        scale = 1 / math.sqrt(shape.head_dim)
        q = c.queries(1)
        want, bound = c.want(q, [L], scale)
        assert torch.isnan(want).any() and not torch.isnan(want).all()
        assert (ekv.ekv_attn_decode_plan(c.pool.handle, 1, c.tables.shape[1])[1] > 1) == (L == 2500)
        check(c.pool.attn_decode(0, q.to(DEV), c.tables, c.lens, scale), want, bound, "decode")
        static = torch.empty_like(q, device=DEV)
        ekv.ekv_attn_decode_static_scratch(c.pool.handle, 0, q.to(DEV), static, c.tables, c.lens, scale)
        check(static, want, bound, "static scratch")
        for n in sorted({1, min(L, 7), min(L, 300)}):
            q = c.queries(n)
            cu = torch.tensor([0, n], dtype=torch.int32)
            want, bound = c.want(q, torch.arange(L - n, L) + 1, scale)
            check(c.pool.attn_prefill_chunk(0, q.to(DEV), c.tables, cu.to(DEV), cu, c.lens, scale), want, bound, f"{n} rows")
        assert c.pool.poll_status() == ekv.Status.OK


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("L", [1, 40, 2500])
def test_rows_of_nan_in_decode(dtype, L):
    """A query with a NaN, and a sequence whose every key is NaN: no range has a maximum, and the row is NaN all the same."""
    shape = I.TINY
    c = Cache(dtype, shape, L, 3, [("K", t, 0, 9, math.nan) for t in range(L)])
    with c.pool:
        q = c.queries(1)
        q[0, 3, 17] = math.nan
        want, bound = c.want(q, [L], 0.125)
        assert torch.isnan(want[0, [0, 1, 3]]).all() and not torch.isnan(want[0, 2]).any()
        check(c.pool.attn_decode(0, q.to(DEV), c.tables, c.lens, 0.125), want, bound)
        # and rows without a key, or with skipped ones only, stay 0
        assert (c.pool.attn_decode(0, c.queries(1).to(DEV), c.tables, torch.zeros_like(c.lens), 0.125) == 0).all()
        assert c.pool.poll_status() == ekv.Status.OK
        none = c.pool.attn_decode(0, c.queries(1).to(DEV), torch.full_like(c.tables, -1), c.lens, 0.125)
        assert (none == 0).all() and c.pool.poll_status() == ekv.Status.ERR_BLOCK_OOB


def spoiled_pair(dtype, shape, L, seed, where, value=math.nan):
    """The same cache with 0 and with `value` in some elements of V (so that scales and all other codes are equal)."""
    return [Cache(dtype, shape, L, seed, [("V", t, h, x, y) for t, h, x in where]) for y in (0.0, value)]


def nan_mask(shape, where, limits):
    """[rows, Hq, D]: a row's channel is NaN if it sees a key whose element is."""
    mask = torch.zeros(len(limits), shape.num_q_heads, shape.head_dim, dtype=torch.bool)
    G = shape.num_q_heads // shape.num_kv_heads
    for t, h, x in where:
        mask[torch.as_tensor(limits) > t, h * G:(h + 1) * G, x] = True
    return mask


def same_but_for(clean, got, mask, bound=None):
    """The clean result, NaN exactly where the mask says: bit for bit, or each within `bound` of what both approximate."""
    clean, got = clean.cpu(), got.cpu()
    assert torch.isfinite(clean.float()).all()
    nan = torch.isnan(got)
    assert torch.equal(nan, mask), f"{int((nan & ~mask).sum())} NaN too many, {int((mask & ~nan).sum())} too few"
    if bound is None:
        assert torch.equal(got[~mask], clean[~mask])
    else:
        assert ((got.double() - clean.double()).abs() <= 2 * bound)[~mask].all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("L", [1, 40, 2500])
def test_a_value_that_is_not_finite_in_decode(dtype, L):
    shape = I.LLAMA8B
    where = [(L - 1, 2, 0), (L // 2, 7, 127), (0, 3, 64)]
    pair = spoiled_pair(dtype, shape, L, 11, where)
    q = pair[0].queries(1).to(DEV)
    clean, got = (c.pool.attn_decode(0, q, c.tables, c.lens, 0.09) for c in pair)
    same_but_for(clean, got, nan_mask(shape, where, [L]))
    for c in pair:
        c.pool.close()


@pytest.mark.parametrize("shape", [I.TINY, I.LLAMA8B, I.Shape(28, 4, 128), I.Shape(5, 1, 64), I.Shape(8, 8, 64)], ids=str)
@pytest.mark.parametrize("L,n", [(700, 700), (700, 129), (333, 100), (3000, 40), (9000, 70), (150, 33), (129, 1), (2000, 2), (45, 3), (6000, 8), (700, 31),
                                 (5, 5), (4001, 32)])
def test_a_value_that_is_not_finite_does_not_reach_rows_before_it(shape, L, n):
    """Rows that share a tile with a NaN of a later key stay finite, rows from it on have it in its channel.  Chunks of one and of
    several items of rows, slots with rows or keys of their own, keys cut over clusters; a NaN code past the end is nobody's."""
    rng = np.random.default_rng(L * 1000 + n)
    at = sorted({L - n, L - 1, L - n + n // 2, max(0, L - n - 1), L // 3, *(int(x) for x in rng.integers(L - n, L, 5))})
    where = [(t, int(rng.integers(shape.num_kv_heads)), int(rng.integers(shape.head_dim))) for t in at]
    pair = spoiled_pair(ekv.EKV_E4M3, shape, L, L + n, where)
    q, cu = pair[0].queries(n).to(DEV), torch.tensor([0, n], dtype=torch.int32)
    outs = [c.pool.attn_prefill_chunk(0, q, c.tables, cu.to(DEV), cu, c.lens, 0.09) for c in pair]
    limits = torch.arange(L - n, L) + 1
    # a request of up to 32 rows a kv-head that meets such a value is computed anew, its sums in another order
    few = n * (shape.num_q_heads // shape.num_kv_heads) <= 32
    same_but_for(*outs, nan_mask(shape, where, limits), pair[0].want(q.cpu(), limits, 0.09)[1] if few else None)
    for c in pair:
        assert c.pool.poll_status() == ekv.Status.OK
        c.pool.close()


@pytest.mark.parametrize("shape", [I.LLAMA8B, I.Shape(8, 2, 64)], ids=str)
def test_one_prompt_with_nan_values_among_many(shape):
    """Several items a CTA, one after the other: those after a spoiled one are as they would be; prompts, drafts and single rows in
    one call, captured and replayed."""
    rng = np.random.default_rng(17)
    lens = [int(x) for x in rng.integers(1, 260, 90)]
    chunks = [L if r % 3 else min(L, 1 + r % 8) for r, L in enumerate(lens)]
    starts = np.concatenate([[0], np.cumsum([-(-L // 16) for L in lens])])
    where, spoil = [], []
    for r in (5, 6, 33, 60, 88):                            # prompts and short chunks
        for _ in range(3):
            t, h, x = int(rng.integers(lens[r])), int(rng.integers(shape.num_kv_heads)), int(rng.integers(shape.head_dim))
            where.append((r, t, h, x))
            spoil.append((int(starts[r]) * 16 + t, h, x))
    pair = spoiled_pair(ekv.EKV_E4M3, shape, int(starts[-1]) * 16, 19, spoil)
    width = int(np.diff(starts).max())
    cu = torch.tensor(np.concatenate([[0], np.cumsum(chunks)]), dtype=torch.int32)
    q, outs = pair[0].queries(int(cu[-1])).to(DEV), []
    d_lens, d_cu = torch.tensor(lens, dtype=torch.int32, device=DEV), cu.to(DEV)
    for c in pair:
        tables = torch.full((len(lens), width), -1, dtype=torch.int32, device=DEV)
        for r in range(len(lens)):
            tables[r, :starts[r + 1] - starts[r]] = c.tables[0, starts[r]:starts[r + 1]]
        out = torch.full_like(q, 7.0)
        c.pool.attn_prefill_chunk(0, q, tables, d_cu, cu, d_lens, 0.09, out=out)
        first, graph = out.clone(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            c.pool.attn_prefill_chunk(0, q, tables, d_cu, cu, d_lens, 0.09, out=out)
        for _ in range(3):
            out.fill_(7.0)
            graph.replay()
            assert torch.equal(out.view(torch.int16), first.view(torch.int16))
        outs.append(first)
        assert c.pool.poll_status() == ekv.Status.OK
    mask = torch.cat([nan_mask(shape, [w[1:] for w in where if w[0] == r], torch.arange(L - n, L) + 1) for r, (L, n) in enumerate(zip(lens, chunks))])
    assert mask.any()
    exact = torch.ones(len(mask), dtype=torch.bool)
    G, c = shape.num_q_heads // shape.num_kv_heads, pair[0]
    for r, (L, n) in enumerate(zip(lens, chunks)):
        a, b = int(cu[r]), int(cu[r + 1])
        if n * G > 32 or not any(w[0] == r and w[1] > L - n for w in where):
            continue
        exact[a:b] = False                                  # few rows: computed anew
        keys = slice(int(starts[r]) * 16, int(starts[r]) * 16 + L)
        bound = M.attention(q[a:b].double().cpu(), c.K[keys], c.V[keys], torch.arange(L - n, L) + 1, 0.09, c.sv[keys])[1]
        same_but_for(*(o[a:b] for o in outs), mask[a:b], bound)
    same_but_for(*(o.cpu()[exact] for o in outs), mask[exact])
