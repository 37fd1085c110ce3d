"""Prefill with modified scores: what stands in the cache at keys that no row sees changes not a bit of the result."""
import pytest
import torch

from scored_model import DEV, Batch, check, slopes_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("mods", [{"cap": 30.0}, {"cap": 30.0, "bias": True}, {"cap": 5.0, "window": 40}, {"window": 40}, {"bias": True}, {"cap": 1e6}], ids=str)
@pytest.mark.parametrize("Hq,Hk,D,past,new", [(4, 2, 64, [0, 200, 500], [90, 40, 300]), (7, 1, 128, [100, 0], [40, 233]), (8, 2, 128, [5003], [3])], ids=str)
def test_bits_do_not_depend_on_keys_that_nobody_sees(Hq, Hk, D, past, new, mods):
    b = Batch(Hq, Hk, D, past, new, seed=61, magnitude=2.0, stale=False)
    cap, window, slopes = mods.get("cap", 0.0), mods.get("window", 0), slopes_of(Hq) if "bias" in mods else None
    call = lambda: b.pool.attn_prefill_chunk_scored(0, b.q, b.tables, b.cu, b.cu_host, b.seq_lens, b.scale, cap=cap, window=window, slopes=slopes)
    unseen = []                                                     # (block, slot) behind a sequence's end and in front of its first row's window
    for r, (a, n) in enumerate(zip(b.past, b.lens)):
        for key in [*range(n, -(-n // 16) * 16), *range(0, max(0, a - window + 1) if window else 0)]:
            unseen.append((int(b.tables_host[r, key // 16]), key % 16))
    blk, slot = torch.tensor(unseen, device=DEV).T
    got = []
    for value in (0.0, 1.0, 1e4, 1e30, float("inf"), float("nan")):
        b.cache[blk, :, :, slot] = value
        got.append(call())
        assert torch.equal(got[0], got[-1]), value
    b.cache[blk, :, :, slot] = 0.0                                  # (the model multiplies them by 0)
    check(got[0], b.model(cap=cap, window=window, slopes=slopes))
