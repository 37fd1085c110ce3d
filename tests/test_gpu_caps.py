"""Caps far above the scores: cap * tanh(score / cap) keeps the score's own accuracy, not the cap's.  Decode and prefill against float64."""
import math

import pytest
import torch

import paper_2608_23658_b200 as ekv  # noqa: F401
from scored_model import BF16, DEV, Batch, slopes_of

pytestmark = pytest.mark.gpu
CAPS = [0.5, 30.0, 3e3, 1e4, 1e5, 1e6, 1e7, 1e10, 1e30, 1e38, 3.4e38]


def model(b, cap=0.0, scale=None, slopes=None, window=0):
    """(result, bound) [T, Hq, D].  A score is a sum of D products in fp32 (2^-23 D of the sum of magnitudes); its cap costs 2^-19 of the CAPPED score: a polynomial with
    a relative error below 2^-20, or 1 - 2 / (e^2y + 1) with some 2^-22 of 1 where tanh is above 0.55; the argument's rounding passes through with a factor of at
    most 1.  Weights and result are rounded to bf16."""
    scale, grp, at = b.scale if scale is None else scale, b.Hq // b.Hk, 0
    out = torch.zeros((b.T, b.Hq, b.D), dtype=torch.float64, device=DEV)
    bound = torch.zeros_like(out)
    for r, (c, n) in enumerate(zip(b.new, b.lens)):
        K, V = b.kv(r)
        p, j = torch.arange(n - c, n, device=DEV)[:, None], torch.arange(n, device=DEV)
        seen = (j <= p) & (j > p - window) if window else j <= p
        for h in range(b.Hq):
            q, k, v = b.q[at:at + c, h].double(), K[h // grp], V[h // grp]
            s = (q @ k.T) * scale
            off = 2.0 ** -23 * b.D * abs(scale) * (q.abs() @ k.abs().T)
            if cap:
                s = cap * torch.tanh(s / cap)
                off = torch.minimum(off, 2 * s.abs()) + 2.0 ** -19 * s.abs()   # (tanh is 1-Lipschitz and saturates)
            if slopes is not None:
                bias = float(slopes[h]) * (p - j).abs().double()
                s, off = s - bias, off + 2.0 ** -22 * bias.clamp(max=200.0)
            s = s.masked_fill(~seen, -math.inf)
            w = torch.softmax(s, -1)
            off = (off * w).sum(-1, keepdim=True) + torch.where(seen & (w > 2.0 ** -30), off, torch.zeros_like(off)).amax(-1, keepdim=True)
            o, mass = w @ v, w @ v.abs()
            out[at:at + c, h] = o
            bound[at:at + c, h] = mass * (2.0 ** -8 + 2 * off + 2.0 ** -16) + o.abs() * 2.0 ** -8 + 1e-30
        at += c
    return out, bound


def call(b, decode, **mods):
    scale = mods.pop("scale", b.scale)
    if decode:
        return b.pool.attn_decode_scored(0, b.q, b.tables, b.seq_lens, scale, **mods)
    return b.pool.attn_prefill_chunk_scored(0, b.q, b.tables, b.cu, b.cu_host, b.seq_lens, scale, **mods)


def check(b, decode, what="", **mods):
    got, (want, bound) = call(b, decode, **mods), model(b, **mods)
    assert torch.isfinite(got).all(), what
    worst = ((got.double() - want).abs() / bound).max().item()
    assert worst <= 1, f"{what}: {worst:.3g} times the bound"
    return got, want, bound


def batch(decode, Hq=4, Hk=2, D=64, seed=31, magnitude=8.0):
    return Batch(Hq, Hk, D, [200, 60, 700], [1, 1, 1], seed=seed, magnitude=magnitude) if decode else Batch(Hq, Hk, D, [200, 0, 0], [40, 160, 300], seed=seed, magnitude=magnitude)


@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("decode", [True, False], ids=["decode", "prefill"])
def test_caps_above_the_scores(decode, bias):
    for Hq, Hk, D in ((4, 2, 64), (7, 1, 128)):
        b = batch(decode, Hq, Hk, D)
        slopes = slopes_of(Hq) if bias else None
        plain = call(b, decode, slopes=slopes).double()
        for cap in CAPS:
            got, want, bound = check(b, decode, f"cap {cap}", cap=cap, slopes=slopes)
            if cap >= 1e7:                                              # tanh(y) is y to 2^-38: no cap at all
                assert ((got.double() - plain).abs() <= 2 * bound).all(), cap


@pytest.mark.parametrize("decode", [True, False], ids=["decode", "prefill"])
def test_caps_above_the_scores_with_a_negative_scale_and_a_window(decode):
    b = batch(decode, seed=32)
    for cap in (50.0, 1e5, 1e30, 3.4e38):
        check(b, decode, f"cap {cap}", cap=cap, scale=-0.1, window=50)


@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("decode", [True, False], ids=["decode", "prefill"])
def test_rows_beside_others_that_are_far_beyond_the_cap(decode, bias):
    b = batch(decode, seed=33)
    b.q[1::3] = (b.q[1::3].float() * 1e7).to(BF16)
    slopes = slopes_of(4) if bias else None
    for cap in (30.0, 1e4, 1e5, 1e6):
        check(b, decode, f"cap {cap}", cap=cap, slopes=slopes)


@pytest.mark.parametrize("decode", [True, False], ids=["decode", "prefill"])
def test_large_caps_beside_slots_that_hold_anything(decode):
    b = batch(decode, seed=34)
    for r, n in enumerate(b.lens):
        if n % 16:
            b.cache[int(b.tables[r, n // 16]), :, :, n % 16:] = 1e30
    for cap in (1e4, 1e6):
        check(b, decode, f"cap {cap}", cap=cap)
