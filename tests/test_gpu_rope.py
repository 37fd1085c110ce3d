"""Norm, rotation and KV write in one pass against the formulas in 64 bits: styles, axes, partial rotation, strides, far positions, slots to
skip, 8-bit pools."""
import math

import pytest
import torch

import paper_2608_23658_b200 as ekv

pytestmark = pytest.mark.gpu
DEV, BF16 = "cuda", torch.bfloat16


def plain(x, weight, positions, inv_freq, axes, adjacent, eps, offset, factor):
    """float64: x [T, H, D]."""
    x, pairs = x.double(), inv_freq.numel()
    if weight is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * (offset + weight.double())
    if pairs == 0:
        return x
    pos = positions.double().view(-1, x.shape[0])[torch.tensor(axes or [0] * pairs, device=x.device)].T   # [T, pairs]
    t = pos * inv_freq.double()
    c, s = factor * torch.cos(t)[:, None], factor * torch.sin(t)[:, None]
    r = x[..., :2 * pairs]
    a, b = (r[..., 0::2], r[..., 1::2]) if adjacent else (r[..., :pairs], r[..., pairs:])
    u, w = a * c - b * s, a * s + b * c
    r = torch.stack([u, w], -1).flatten(-2) if adjacent else torch.cat([u, w], -1)
    return torch.cat([r, x[..., 2 * pairs:]], -1)


def bound(x, weight, want, inv_freq, eps, offset, factor):
    """What fp32 arithmetic and one rounding to bf16 may be off by.  Rounding: 2^-8 of the value.  fp32: the norm's factor, the weight, the
    sines (some 2^-21 of 1 with their argument's last bits) and the sum of two products: 2^-19 of the larger of the pair, which is at most the row's largest magnitude."""
    top = x.double().abs().amax(-1, keepdim=True)
    if weight is not None:
        top = top / torch.sqrt((x.double() ** 2).mean(-1, keepdim=True) + eps) * (offset + weight.double()).abs().amax()
    return want.abs() * 2.0 ** -8 + top * max(1.0, abs(factor)) * 2.0 ** -19 + 1e-38


def make(T, Hq, Hk, D, rot, axes, norm, seed=0, far=100000, fused=True, dtype=ekv.EKV_BF16):
    g = torch.Generator(device=DEV).manual_seed(seed)
    nb = (T + 15) // 16 + 3
    pool = ekv.Pool(num_q_heads=Hq, num_kv_heads=Hk, head_dim=D, base_blocks=nb, dtype=dtype)
    width = Hq + 2 * Hk
    rows = torch.randn((T, width + (0 if fused else 3), D), generator=g, device=DEV).to(BF16)
    q, k, v = rows[:, :Hq], rows[:, Hq:Hq + Hk], rows[:, Hq + Hk:width]
    slots = torch.randperm(nb * 16, generator=g, device=DEV)[:T].to(torch.int64)
    positions = torch.randint(0, far, (axes, T), generator=g, device=DEV, dtype=torch.int32)
    pair_axis = [i * axes // max(rot // 2, 1) for i in range(rot // 2)] if axes > 1 else None
    inv_freq = (10000.0 ** (-torch.arange(rot // 2, device=DEV, dtype=torch.float64) / max(rot // 2, 1))).float()
    qw = torch.randn(D, generator=g, device=DEV).to(BF16) if norm else None
    kw = torch.randn(D, generator=g, device=DEV).to(BF16) if norm else None
    return pool, q, k, v, slots, positions if axes > 1 else positions[0], pair_axis, inv_freq, qw, kw


def check(pool, q, k, v, slots, positions, pair_axis, inv_freq, qw, kw, adjacent, eps=1e-6, offset=0.0, factor=1.0, **more):
    before = pool.layer_tensor(0).clone()
    q64, k64, v0 = q.clone(), k.clone(), v.clone()
    out = pool.rope_write_kv(0, q, k, v, positions, inv_freq, slots, q_weight=qw, k_weight=kw, eps=eps, weight_offset=offset, factor=factor,
                             interleaved=adjacent, axes=pair_axis, **more)
    for x, w, got in ((q64, qw, out), (k64, kw, pool.layer_tensor(0)[slots // 16, 0, :, slots % 16])):
        want = plain(x, w, positions, inv_freq, pair_axis, adjacent, eps, offset, factor)
        assert got.shape == want.shape
        err = (got.double() - want).abs()
        assert (err <= bound(x, w, want, inv_freq, eps, offset, factor)).all(), float((err - bound(x, w, want, inv_freq, eps, offset, factor)).max())
    after = pool.layer_tensor(0)
    assert torch.equal(after[slots // 16, 1, :, slots % 16], v0)
    after, before = after.clone(), before
    after[slots // 16, :, :, slots % 16] = before[slots // 16, :, :, slots % 16]
    assert torch.equal(after.view(torch.int16), before.view(torch.int16))      # nothing else changed
    assert pool.poll_status() == ekv.Status.OK
    return out


@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("T,Hq,Hk,D,rot,axes,norm", [
    (1, 4, 2, 64, 64, 1, False), (1, 5, 1, 128, 128, 1, True), (31, 4, 2, 64, 32, 1, True), (17, 28, 4, 128, 128, 3, True),
    (257, 32, 8, 128, 64, 2, True), (40, 6, 2, 128, 6, 3, False), (33, 8, 8, 64, 50, 4, True), (19, 8, 8, 128, 126, 1, True),
    (12, 16, 2, 64, 0, 1, True), (3, 64, 8, 128, 2, 1, False), (5000, 4, 1, 64, 64, 1, True), (9500, 2, 1, 128, 34, 1, False)])
def test_against_the_formulas(T, Hq, Hk, D, rot, axes, norm, adjacent):
    check(*make(T, Hq, Hk, D, rot, axes, norm, seed=T), adjacent)


def test_offset_factor_and_one_norm_alone():
    x = list(make(37, 8, 2, 128, 96, 1, True))
    check(*x, False, eps=1e-3, offset=1.0, factor=1.37)
    check(*x[:8], None, x[9], True, offset=1.0)
    check(*x[:9], None, True)


def test_far_positions_keep_their_angle():
    pool, q, k, v, slots, _, axes, inv_freq, qw, kw = make(64, 4, 2, 64, 64, 1, False)
    positions = torch.arange(64, device=DEV, dtype=torch.int32) * 33554431      # up to 2^31
    check(pool, q, k, v, slots, positions, axes, inv_freq, qw, kw, False)
    check(pool, q, k, v, slots, -positions, axes, inv_freq, qw, kw, True)


def test_rows_apart_and_in_place():
    pool, q, k, v, *rest = make(50, 4, 2, 128, 128, 1, True, fused=False)
    out = check(pool, q, k, v, *rest, False)
    want = out.clone()
    again = check(pool, q, k, v, *rest, False, q_out=q)                        # the projection's own rows
    assert again.data_ptr() == q.data_ptr() and torch.equal(again, want)


def test_zero_rows_and_values_that_are_not_finite():
    pool, q, k, v, slots, positions, axes, inv_freq, qw, kw = make(20, 4, 2, 64, 64, 1, True)
    q[3], k[5, 1] = 0, 0
    v[7, 0, 3], v[8, 1, 60] = float("nan"), float("inf")
    q[4, 1, 10] = float("nan")                                                  # reaches its own head's row only
    clean = torch.ones(20, 4, dtype=torch.bool, device=DEV)
    clean[4, 1] = False
    out = pool.rope_write_kv(0, q, k, v, positions, inv_freq, slots, q_weight=qw, k_weight=kw)
    assert torch.isnan(out[4, 1]).all() and torch.isfinite(out[clean]).all() and (out[3] == 0).all()
    kv = pool.layer_tensor(0)[slots // 16, :, :, slots % 16]
    assert (kv[5, 0, 1] == 0).all() and torch.isfinite(kv[:, 0]).all()
    assert torch.equal(kv[:, 1].contiguous().view(torch.int16), v.contiguous().view(torch.int16))


def test_slots_to_skip_and_slots_out_of_range():
    pool, q, k, v, slots, positions, axes, inv_freq, qw, kw = make(33, 4, 2, 64, 64, 1, False)
    want = pool.rope_write_kv(0, q, k, v, positions, inv_freq, slots)
    pool.layer_tensor(0).fill_(7)
    odd = slots.clone()
    odd[::3] = -1
    got = pool.rope_write_kv(0, q, k, v, positions, inv_freq, odd)
    assert torch.equal(got, want) and pool.poll_status() == ekv.Status.OK
    skipped = slots[::3]
    assert (pool.layer_tensor(0)[skipped // 16, :, :, skipped % 16] == 7).all()
    odd[1] = int(pool.info.live_blocks) * 16
    got = pool.rope_write_kv(0, q, k, v, positions, inv_freq, odd)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and pool.poll_status() == ekv.Status.ERR_BLOCK_OOB
    none = torch.empty(0, dtype=torch.int64, device=DEV)
    assert pool.rope_write_kv(0, q[:0], k[:0], v[:0], positions[:0], inv_freq, none).shape == (0, 4, 64)


@pytest.mark.parametrize("T", [1, 50, 1500])
def test_8bit_pools_quantise_the_finished_keys(T):
    x = make(T, 4, 2, 128, 64, 1, True, dtype=ekv.EKV_E4M3)
    pool, q, k, v, slots, positions, axes, inv_freq, qw, kw = x
    slots = torch.arange(T, device=DEV)
    other = ekv.Pool(num_q_heads=4, num_kv_heads=2, head_dim=128, base_blocks=int(pool.info.base_blocks), dtype=ekv.EKV_E4M3)
    k_out = torch.empty((T, 2, 128), dtype=BF16, device=DEV)
    out = pool.rope_write_kv(0, q, k, v, positions, inv_freq, slots, q_weight=qw, k_weight=kw, k_out=k_out)
    for rows, w, got in ((q, qw, out), (k, kw, k_out)):
        want = plain(rows, w, positions, inv_freq, None, False, 1e-6, 0.0, 1.0)
        assert ((got.double() - want).abs() <= bound(rows, w, want, inv_freq, 1e-6, 0.0, 1.0)).all()
    other.write_kv(0, k_out, v.contiguous(), slots)
    used = (T + 15) // 16
    assert torch.equal(pool.layer_scales(0)[:used], other.layer_scales(0)[:used])
    for a, b in zip(pool.read_kv(0, slots), other.read_kv(0, slots)):
        assert torch.equal(a, b)


def test_on_a_stream_of_its_own_and_replayed():
    pool, q, k, v, slots, positions, axes, inv_freq, qw, kw = make(40, 8, 2, 128, 128, 1, True)
    want = pool.rope_write_kv(0, q, k, v, positions, inv_freq, slots, q_weight=qw, k_weight=kw)
    cache = pool.layer_tensor(0).clone()
    out = torch.empty_like(want)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        pool.rope_write_kv(0, q, k, v, positions, inv_freq, slots, q_weight=qw, k_weight=kw, q_out=out)
    pool.layer_tensor(0)[slots // 16, :, :, slots % 16] = 0
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want) and torch.equal(pool.layer_tensor(0).view(torch.int16), cache.view(torch.int16))
    slots2 = torch.flip(slots, (0,))
    with torch.cuda.stream(side):
        pool.rope_write_kv(0, q, k, v, positions, inv_freq, slots2, q_weight=qw, k_weight=kw, q_out=out)
    side.synchronize()
    assert torch.equal(out, want)


def test_refusals():
    pool, q, k, v, slots, positions, axes, inv_freq, qw, kw = make(6, 4, 2, 64, 64, 2, True)
    call = lambda pool=pool, layer=0, q=q, k=k, v=v, axes=axes, inv_freq=inv_freq, **more: pool.rope_write_kv(
        layer, q, k, v, positions, inv_freq, slots, axes=axes, **{"q_weight": qw, "k_weight": kw, **more})
    before = pool.layer_tensor(0).clone()
    wide = torch.zeros(6 * 8 * 64 + 8, dtype=BF16, device=DEV)
    apart = lambda heads, stride, first=0: torch.as_strided(wide, (6, heads, 64), (stride, 64, 1), first)
    long = torch.ones(33, device=DEV)
    for bad in ({"layer": 1}, {"layer": -1}, {"axes": [0] * 31 + [2]}, {"eps": -1.0}, {"eps": float("nan")}, {"inv_freq": long, "axes": [0] * 33},
                {"q": apart(4, 64)}, {"k": apart(2, 64)}, {"v": apart(2, 64)}, {"q_out": apart(4, 192)},      # tokens over one another
                {"q": apart(4, 256), "q_out": apart(4, 320)},
                {"q": apart(4, 260)}, {"k": apart(2, 132)}, {"v": apart(2, 256, 4)}, {"q_out": apart(4, 256, 1)},   # off 16 bytes
                {"k_weight": torch.zeros(72, dtype=BF16, device=DEV)[1:65]}, {"k_out": torch.empty((6, 2, 64), dtype=BF16, device=DEV)}):
        with pytest.raises(ekv.EkvError) as e:
            call(**bad)
        assert e.value.status == ekv.Status.ERR_INVALID, bad
    torch.cuda.synchronize()
    assert torch.equal(pool.layer_tensor(0).view(torch.int16), before.view(torch.int16)) and not wide.any()
    call()


def test_the_keys_of_an_8bit_pool_pass_through_memory_of_the_calls_stream():
    T, side = 400, torch.cuda.Stream()
    pool, q, k, v, slots, positions, axes, inv_freq, qw, kw = make(T, 4, 2, 128, 128, 1, True, dtype=ekv.EKV_E4M3)
    slots, out = torch.arange(T, device=DEV), torch.empty((T, 4, 128), dtype=BF16, device=DEV)
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    before = torch.cuda.memory_stats()["allocation.all.allocated"]
    pool.rope_write_kv(0, q, k, v, positions, inv_freq, slots, q_weight=qw, k_weight=kw, q_out=out, stream=side)
    assert torch.cuda.memory_stats()["allocation.all.allocated"] == before + 1
    assert any(s["stream"] == side.cuda_stream for s in torch.cuda.memory_snapshot())
    side.synchronize()
    got = pool.read_kv(0, slots)
    pool.rope_write_kv(0, q, k, v, positions, inv_freq, slots, q_weight=qw, k_weight=kw, q_out=out)
    assert all(torch.equal(a, b) for a, b in zip(got, pool.read_kv(0, slots)))
