"""The operators as a model's layers use them together: rotation and write, prefill, decode over a shared prefix, with the step's tables made on the
GPU; and a windowed, capped layer over the same requests."""
import math

import pytest
import torch

import paper_2608_23658_b200 as ekv
from scored_model import BF16, DEV, BS, Batch, check

pytestmark = pytest.mark.gpu
Hq, Hk, D, EPS = 8, 2, 64, 1e-6


class Requests:
    """Requests over one pool whose first `prefix` tokens are those of the first one; what they hold is read back for the model."""

    def __init__(self, n, prefix, room):
        g = torch.Generator(device=DEV).manual_seed(n)
        shared, own = prefix // BS, -(-room // BS) + 1
        self.n, self.prefix, width = n, prefix, shared + own
        self.pool = ekv.Pool(num_q_heads=Hq, num_kv_heads=Hk, head_dim=D, base_blocks=shared + n * own + 9)
        self.cache = self.pool.layer_tensor(0)
        self.cache.fill_(float("nan"))                                      # what was never written
        self.tables = torch.full((n, width), -1, dtype=torch.int32, device=DEV)
        self.tables[:, :shared] = torch.arange(shared, dtype=torch.int32, device=DEV)
        self.free = (shared + torch.randperm(n * own, generator=g, device=DEV)).to(torch.int32)
        self.cursor = torch.zeros(1, dtype=torch.int32, device=DEV)
        self.lens = torch.full((n,), prefix, dtype=torch.int32, device=DEV)
        self.slots = torch.empty(n, dtype=torch.int64, device=DEV)
        self.cu = torch.empty(n + 1, dtype=torch.int32, device=DEV)
        self.one = torch.ones(n, dtype=torch.int32, device=DEV)
        self.inv_freq = (10000.0 ** (-torch.arange(D // 2, device=DEV, dtype=torch.float64) / (D // 2))).float()
        self.qw, self.kw = (1 + 0.1 * torch.randn(2, D, generator=g, device=DEV)).to(BF16)
        self.g, self.scale = g, 1 / math.sqrt(D)

    def rows(self, T):
        x = torch.randn((T, (Hq + 2 * Hk) * D), generator=self.g, device=DEV).to(BF16).view(T, Hq + 2 * Hk, D)
        return x[:, :Hq], x[:, Hq:Hq + Hk], x[:, Hq + Hk:]

    def rotate(self, q, k, v, positions, slots, **more):
        return self.pool.rope_write_kv(0, q, k, v, positions, self.inv_freq, slots, q_weight=self.qw, k_weight=self.kw, eps=EPS, **more)

    def model(self, q, **mods):
        """The attention model over what the cache holds now, for one row a request."""
        b = Batch.__new__(Batch)
        b.Hq, b.Hk, b.D, b.T, b.q, b.cache, b.scale = Hq, Hk, D, self.n, q, self.cache, self.scale
        b.lens = self.lens.tolist()
        b.new, b.tables_host = [1] * self.n, self.tables.cpu().numpy()
        return b.model(**mods)


@pytest.mark.parametrize("n,prefix", [(5, 64), (6, 12000), (6, 36000)])
def test_samples_of_one_prompt(n, prefix):
    r = Requests(n, prefix, room=40)
    q, k, v = r.rows(prefix)
    slots = torch.arange(prefix, device=DEV)
    q = r.rotate(q, k, v, torch.arange(prefix, dtype=torch.int32, device=DEV), slots)
    cu = torch.tensor([0, prefix], dtype=torch.int32)
    out = r.pool.attn_prefill_chunk_scored(0, q, r.tables[:1].contiguous(), cu.to(DEV), cu, r.lens[:1].contiguous(), r.scale)
    again = r.pool.attn_prefill_chunk(0, q, r.tables[:1].contiguous(), cu.to(DEV), cu, r.lens[:1].contiguous(), r.scale)
    assert torch.isfinite(out).all() and (out.float() - again.float()).abs().max() < 0.05
    starts, shared = torch.tensor([0, n], dtype=torch.int32), torch.tensor([prefix], dtype=torch.int32)

    # one captured step, replayed while the requests grow: tables, rotation and write, attention
    q, k, v = r.rows(n)
    q_out, out = torch.empty((n, Hq, D), dtype=BF16, device=DEV), torch.empty((n, Hq, D), dtype=BF16, device=DEV)
    positions = torch.empty(n, dtype=torch.int32, device=DEV)
    far = torch.empty_like(out)

    def step():
        positions.copy_(r.lens)
        r.pool.extend_tables(r.one, r.lens, r.tables, r.free, r.cursor, r.slots, r.cu)
        r.rotate(q, k, v, positions, r.slots, q_out=q_out)
        r.pool.attn_decode_shared(0, q_out, r.tables, r.lens, starts, shared, r.scale, out=out)
        r.pool.attn_decode_scored(0, q_out, r.tables, r.lens, r.scale, cap=20.0, window=50, out=far)

    step()
    check(out, r.model(q_out))
    check(far, r.model(q_out, cap=20.0, window=50))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step()
    for _ in range(20):
        q.copy_(torch.randn(q.shape, generator=r.g, device=DEV))
        k.copy_(torch.randn(k.shape, generator=r.g, device=DEV))
        graph.replay()
    torch.cuda.synchronize()
    assert r.lens.tolist() == [prefix + 21] * n and r.pool.poll_status() == ekv.Status.OK
    check(out, r.model(q_out))
    check(far, r.model(q_out, cap=20.0, window=50))


def test_a_prompt_in_chunks_is_a_prompt_at_once():
    mods = dict(cap=15.0, window=90, prefix_lens=torch.tensor([40], dtype=torch.int32, device=DEV))
    b = Batch(Hq, Hk, D, [0], [300], seed=3)
    whole = b.pool.attn_prefill_chunk_scored(0, b.q, b.tables, b.cu, b.cu_host, b.seq_lens, b.scale, **mods)
    check(whole, b.model(cap=15.0, window=90, prefix=[40]))
    parts = []
    for a, e in ((0, 64), (64, 65), (65, 200), (200, 300)):
        cu = torch.tensor([0, e - a], dtype=torch.int32)
        parts.append(b.pool.attn_prefill_chunk_scored(0, b.q[a:e], b.tables, cu.to(DEV), cu, torch.tensor([e], dtype=torch.int32, device=DEV), b.scale, **mods))
    want, bound = b.model(cap=15.0, window=90, prefix=[40])
    assert ((torch.cat(parts).double() - want).abs() <= bound).all()
    last = b.pool.attn_decode_scored(0, b.q[299:], b.tables, b.seq_lens, b.scale, **mods)
    assert ((last.double() - want[299:]).abs() <= bound[299:]).all()
