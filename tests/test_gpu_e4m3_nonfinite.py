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
