"""Arguments that the Python entry points refuse before anything is launched (no GPU needed)."""
import pytest
import torch

import paper_2608_23658_b200 as ekv


class OnGpu(torch.Tensor):
    """A tensor that says it is on the GPU, so that only what else is wrong with it is refused."""

    def get_device(self):
        return 0


def gpu(*shape, dtype=torch.int32):
    return torch.zeros(shape, dtype=dtype).as_subclass(OnGpu)


@pytest.fixture
def calls(monkeypatch):
    """What reaches the library, whose calls are replaced."""
    from paper_2608_23658_b200 import _binding as B
    seen = []

    class Lib:
        def __getattr__(self, name):
            return lambda *args: seen.append((name, *args)) or 0

    monkeypatch.setattr(B, "load_library", lambda: Lib())
    return seen


def a_pool():
    pool = ekv.Pool.__new__(ekv.Pool)
    pool.device, pool.num_kv_heads, pool.head_dim, pool.handle = torch.device("cuda", 0), 2, 64, None
    return pool


def test_read_kv_refuses_outputs_that_it_would_write_past(calls):
    pool, slots, bf16 = a_pool(), gpu(5, dtype=torch.int64), torch.bfloat16
    k, v = gpu(5, 2, 64, dtype=bf16), gpu(5, 2, 64, dtype=bf16)
    pool.read_kv(0, slots, k, v, stream=0)
    pool.read_kv(0, slots, k.view(5, 128), v.view(5, 128), stream=0)
    assert calls == [("ekv_read_kv", None, 0, k.data_ptr(), v.data_ptr(), slots.data_ptr(), 5, 0)] * 2
    calls.clear()
    bad = [gpu(4, 2, 64, dtype=bf16), gpu(5, 1, 64, dtype=bf16), gpu(5, 2, 32, dtype=bf16), gpu(5, 2, 64, dtype=torch.float8_e4m3fn),
           gpu(5, 2, 64, dtype=torch.float32), gpu(5, 64, 2, dtype=bf16).transpose(1, 2), gpu(10, 64, dtype=bf16), torch.zeros(5, 2, 64, dtype=bf16)]
    for b in bad:
        for args in ((b, v), (k, b), (b, b)):
            with pytest.raises(ValueError):
                pool.read_kv(0, slots, *args, stream=0)
    for b in (bad[0], *bad[3:]):
        for args in ((b, v), (k, b)):
            with pytest.raises(ValueError):
                ekv.ekv_read_kv(None, 0, *args, slots, stream=0)
    for b in (gpu(5), gpu(5, dtype=torch.float64), gpu(10, dtype=torch.int64)[::2], torch.zeros(5, dtype=torch.int64)):
        with pytest.raises(ValueError):
            pool.read_kv(0, b, k, v, stream=0)
    assert not calls


def test_extend_tables_refuses_what_is_not_int32(calls):
    pool, R, width = a_pool(), 3, 7
    good = dict(new_tokens=gpu(R), seq_lens=gpu(R), block_tables=gpu(R, width), free_ids=gpu(9), free_cursor=gpu(1),
                slot_mapping=gpu(20, dtype=torch.int64), cu_q_lens=gpu(R + 1), seq_lens_out=gpu(R), free_cursor_out=gpu(1))
    pool.extend_tables(**good, stream=0)
    at = {name: t.data_ptr() for name, t in good.items()}
    assert calls == [("ekv_extend_tables", None, at["new_tokens"], at["seq_lens"], R, at["block_tables"], width, at["free_ids"], 9,
                      at["free_cursor"], at["slot_mapping"], 20, at["cu_q_lens"], at["seq_lens_out"], at["free_cursor_out"], 0)]
    calls.clear()
    for name, t in good.items():
        other = torch.int32 if name == "slot_mapping" else torch.int64
        bad = [t.float(), t.to(other), torch.zeros(t.shape, dtype=t.dtype)]
        if name == "slot_mapping":
            bad.append(gpu(20, dtype=torch.float64))
        if name not in ("free_ids", "slot_mapping"):
            bad.append(t[:-1].contiguous())
        if t.numel() > 1:
            bad.append(torch.cat([t, t], -1)[..., ::2])
        if name == "block_tables":
            bad.append(t.view(-1))
        for b in bad:
            with pytest.raises(ValueError):
                pool.extend_tables(**{**good, name: b}, stream=0)
    assert not calls
