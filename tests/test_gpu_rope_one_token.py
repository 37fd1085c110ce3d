"""The distance between tokens says nothing where there is one: a tensor of one token may have any."""
import pytest
import torch

import paper_2608_23658_b200 as ekv

pytestmark = pytest.mark.gpu
DEV, BF16 = "cuda", torch.bfloat16


@pytest.mark.parametrize("stride", [0, 1, 7, 64, 100003])
@pytest.mark.parametrize("dtype", [ekv.EKV_BF16, ekv.EKV_E4M3])
def test_one_token_with_any_stride(dtype, stride):
    pool = ekv.Pool(num_q_heads=4, num_kv_heads=2, head_dim=64, base_blocks=8, dtype=dtype)
    g = torch.Generator(device=DEV).manual_seed(91)
    rows = torch.randn((1, 8, 64), generator=g, device=DEV).to(BF16)
    q, k, v = (x.clone() for x in (rows[:, :4], rows[:, 4:6], rows[:, 6:]))
    position, inv_freq, slot = torch.tensor([77], dtype=torch.int32, device=DEV), torch.rand(32, generator=g, device=DEV), torch.tensor([21], device=DEV)
    want = pool.rope_write_kv(0, q, k, v, position, inv_freq, slot)
    kv = [x.clone() for x in pool.read_kv(0, slot)]
    odd = lambda x: x.as_strided(x.shape, (stride, 64, 1))
    out = odd(torch.empty_like(q))
    pool.layer_tensor(0).view(torch.uint8).zero_()
    got = pool.rope_write_kv(0, odd(q), odd(k), odd(v), position, inv_freq, slot, q_out=out)
    assert got is out and torch.equal(got, want)
    assert all(torch.equal(a, b) for a, b in zip(pool.read_kv(0, slot), kv))
