"""8-bit pools on a host without a GPU: the models the GPU tests use, pinned against torch's e4m3 conversion; geometry
and refusals through a host model of the VMM calls."""
import numpy as np
import pytest
import torch

import e4m3_model as M
import paper_2608_23658_b200 as ekv
from fake_vmm import FakeVmm

MiB = 1 << 20


@pytest.fixture
def vmm():
    fake = FakeVmm()
    table = fake.table()
    ekv.ekv_set_vmm_backend(table)
    yield fake
    ekv.ekv_set_vmm_backend(None)
    assert fake.violations == []


def test_model_encodes_like_e4m3():
    g = torch.Generator().manual_seed(1)
    x = torch.cat([torch.randn(20000, generator=g) * torch.exp2(torch.rand(20000, generator=g) * 24 - 14),
                   torch.arange(-448, 449, 0.5), torch.arange(0, 64) * 2.0 ** -11]).clamp(-448, 448).double()
    want = x.float().to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(M.encode(x.numpy()), want)
    every = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(M.CODE_VALUE, every, equal_nan=True)


def test_model_scale_is_the_smallest_that_fits():
    for a in [0.0, 1e-40, 2.0 ** -112 * 448, 1.0, 447.9, 448.0, 448.1, 449.0, 1e30, 3.3895e38]:
        s = M.scale_of(a)
        assert a <= 448 * s
        assert s == 2.0 ** M.E_LO or a > 448 * s / 2


def test_model_write_keeps_raises_and_restarts():
    c = M.Cache(2, 1, 64)
    one = np.ones((1, 1, 64))
    c.write(one, one, [0])
    c.write(one * 1000, one * 2, [1])
    k, v = c.rows([0, 1])
    assert np.array_equal(k[0], one[0]) and k[1, 0, 0] == 1024.0 and np.array_equal(v[1], 2 * one[0])  # 1000 lies between 960 and 1024
    assert c.scales[0, 0, 0] == 4.0
    c.write(one, one, [0])  # the first slot again: the block starts anew
    assert c.scales[0, 0, 0] == 2.0 ** -8


def test_geometry_and_refusals(vmm):
    args = dict(num_q_heads=32, num_kv_heads=8, head_dim=128, base_blocks=100, elastic_blocks=40)
    pool = ekv.ekv_pool_create(dtype=ekv.EKV_E4M3, **args)
    info = ekv.ekv_pool_info(pool)
    assert info.block_bytes == 32 * 1024 == info.block_stride_bytes
    assert (info.base_blocks, info.elastic_blocks) == (128, 64) and info.base_bytes == 4 * MiB
    with pytest.raises(ekv.EkvError) as e:
        ekv.ekv_layer_scales(pool, 0)            # no device state behind a replacement backend
    assert e.value.status == ekv.Status.ERR_STATE
    for call in (lambda: ekv.load_library().ekv_write_kv(pool, 0, None, None, None, 0, None),
                 lambda: ekv.load_library().ekv_read_kv(pool, 0, None, None, None, 0, None),
                 lambda: ekv.load_library().ekv_extend_tables(pool, *[None] * 2, 0, None, 1, None, 0, None, None, 0, *[None] * 4)):
        assert call() == ekv.Status.ERR_STATE
    ekv.ekv_grow(pool, host_only=True)
    assert ekv.ekv_pool_info(pool).live_blocks == 192
    ekv.ekv_shrink(pool, host_only=True)
    ekv.ekv_pool_destroy(pool)
    pool = ekv.ekv_pool_create(dtype=ekv.EKV_E4M3, flags=ekv.EKV_FUSED_RANGE, num_layers=3, **args)
    assert ekv.ekv_pool_info(pool).block_stride_bytes == 3 * 32 * 1024
    ekv.ekv_pool_destroy(pool)
    pool = ekv.ekv_pool_create(**args)
    with pytest.raises(ekv.EkvError) as e:
        ekv.ekv_layer_scales(pool, 0)            # a bf16 pool has none
    assert e.value.status == ekv.Status.ERR_INVALID
    ekv.ekv_pool_destroy(pool)
    for bad in (dict(dtype=2), dict(dtype=-1), dict(dtype=ekv.EKV_E4M3, flags=ekv.EKV_PREFILL_WARP_MMA),
                dict(dtype=ekv.EKV_E4M3, flags=ekv.EKV_PREFILL_ONE_HEAD), dict(dtype=ekv.EKV_E4M3, flags=ekv.EKV_PREFILL_TWO_HEAD)):
        with pytest.raises(ekv.EkvError) as e:
            ekv.ekv_pool_create(**args, **bad)
        assert e.value.status == ekv.Status.ERR_INVALID
    assert not vmm.reserved and not vmm.handles and not vmm.mapped


def test_null_pool_is_refused():
    lib = ekv.load_library()
    assert lib.ekv_read_kv(None, 0, None, None, None, 0, None) == ekv.Status.ERR_INVALID
    assert lib.ekv_extend_tables(None, *[None] * 2, 0, None, 1, None, 0, None, None, 0, *[None] * 4) == ekv.Status.ERR_INVALID
