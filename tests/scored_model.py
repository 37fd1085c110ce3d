"""Test-side model of decode and prefill attention with capped, biased, windowed scores and prefix masks: float64, request by request, from the
definition; and what a kernel with fp32 scores and bf16 weights may be off by."""
import math

import numpy as np
import torch

import paper_2608_23658_b200 as ekv

DEV, BF16, BS = "cuda", torch.bfloat16, 16


class Batch:
    """A bf16 pool with a filled cache and a batch over it.  past[r] cached tokens, new[r] query rows; shared[r]: blocks that request r has from
    request `owner[r]`."""

    def __init__(self, Hq, Hk, D, past, new, seed=0, magnitude=1.0, table_extra=0, share=None, stale=True):
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.Hq, self.Hk, self.D, self.past, self.new = Hq, Hk, D, list(past), list(new)
        self.lens = [a + b for a, b in zip(past, new)]
        need = [-(-x // BS) for x in self.lens]
        share = share or [(r, 0) for r in range(len(need))]
        total = sum(n - s for n, (_, s) in zip(need, share)) + 5
        ids = np.random.RandomState(seed).permutation(total)
        width = max(max(need), 1) + table_extra
        tables, at = np.full((len(need), width), -7, np.int32), 0
        for r, (n, (owner, s)) in enumerate(zip(need, share)):
            tables[r, :s] = tables[owner, :s]
            tables[r, s:n] = ids[at:at + n - s]
            at += n - s
        self.pool = ekv.Pool(num_q_heads=Hq, num_kv_heads=Hk, head_dim=D, base_blocks=total)
        self.cache = self.pool.layer_tensor(0, 0, total)
        self.cache.copy_(torch.randn(self.cache.shape, generator=g, device=DEV).to(BF16))
        if stale:  # slots behind a sequence's end, and blocks nobody has, may hold anything
            self.cache[torch.from_numpy(np.setdiff1d(ids, tables[tables >= 0])).to(DEV)] = float("nan")
            for r, n in enumerate(self.lens):
                if n % BS:
                    self.cache[int(tables[r, n // BS]), :, :, n % BS:] = float("nan")
        self.tables_host = tables
        self.tables = torch.from_numpy(tables.copy()).to(DEV)
        self.seq_lens = torch.tensor(self.lens, dtype=torch.int32, device=DEV)
        self.cu_host = torch.from_numpy(np.concatenate([[0], np.cumsum(new)]).astype(np.int32))
        self.cu = self.cu_host.to(DEV)
        self.T = int(self.cu_host[-1])
        self.q = (torch.randn((self.T, Hq, D), generator=g, device=DEV) * magnitude).to(BF16)
        self.scale = 1 / math.sqrt(D)

    def kv(self, r):
        n = self.lens[r]
        ids = torch.from_numpy(self.tables_host[r, :-(-n // BS)]).to(DEV).long()   # (a test may put ids out of range into the call's table)
        return self.cache[ids].double().permute(1, 2, 0, 3, 4).reshape(2, self.Hk, -1, self.D)[:, :, :n]

    def model(self, scale=None, cap=0.0, window=0, slopes=None, prefix=None, skip=()):
        """(result, bound on a kernel's error) [T, Hq, D] in float64."""
        scale = self.scale if scale is None else scale
        out = torch.zeros((self.T, self.Hq, self.D), dtype=torch.float64, device=DEV)
        bound, grp, at = torch.zeros_like(out), self.Hq // self.Hk, 0
        for r, (c, n) in enumerate(zip(self.new, self.lens)):
            if c == 0 or n == 0 or r in skip:
                at += c
                continue
            K, V = self.kv(r)
            p, j = torch.arange(n - c, n, device=DEV)[:, None], torch.arange(n, device=DEV)
            seen = j <= p
            if window:
                seen &= j > p - window
            if prefix is not None:
                seen |= j < int(prefix[r])
            for h in range(self.Hq):
                q = self.q[at:at + c, h].double()
                s = (q @ K[h // grp].T) * scale
                # fp32 sums of D products, a few more roundings of the score, its cap and its bias
                off = 2.0 ** -23 * self.D * abs(scale) * (q.abs() @ K[h // grp].abs().T) + 2.0 ** -21 * s.abs()
                if cap:
                    s = cap * torch.tanh(s / cap)
                    off = off + 2.0 ** -20 * cap
                if slopes is not None:
                    bias = float(slopes[h]) * (p - j).abs().double()
                    s, off = s - bias, off + 2.0 ** -22 * torch.minimum(bias, torch.full_like(bias, 200.0))
                s = s.masked_fill(~seen, -math.inf)
                w = torch.softmax(s, -1)
                off = (off * w).sum(-1, keepdim=True) + torch.where(seen & (w > 2.0 ** -30), off, torch.zeros_like(off)).amax(-1, keepdim=True)
                o, mass = w @ V[h // grp], w @ V[h // grp].abs()
                out[at:at + c, h] = o
                # weights rounded to bf16 (2^-8 each), the result as well; fp32 statistics and sums
                bound[at:at + c, h] = mass * (2.0 ** -8 + 2 * off + 2.0 ** -16) + o.abs() * 2.0 ** -8 + 1e-30
            at += c
        return out, bound


def check(got, model, what=""):
    want, bound = model
    assert got.shape == want.shape and torch.isfinite(got).all(), what
    err = (got.double() - want).abs()
    worst = (err / bound.clamp(min=1e-30)).max().item()
    assert (err <= bound).all(), f"{what}: {worst:.3g} times the bound, max-abs {err.max().item():.3g}"


def slopes_of(Hq):
    return (2.0 ** (-8.0 * (torch.arange(Hq, dtype=torch.float64) + 1) / Hq)).float().to(DEV)
