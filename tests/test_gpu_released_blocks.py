"""Blocks that a window has passed may have been given back: whatever their table entries hold, no row changes and no error is latched."""
import pytest
import torch

import paper_2608_23658_b200 as ekv
from scored_model import DEV, Batch, check, slopes_of

pytestmark = pytest.mark.gpu


def gone(b, window, prefix=0):
    """(request, block) of the tables that no row of a call sees a key of."""
    for r, (past, n) in enumerate(zip(b.past, b.lens)):
        first = max(0, past - window + 1)
        for block in range(-(-n // 16)):
            if block * 16 >= prefix and block * 16 + 16 <= first:
                yield r, block


@pytest.mark.parametrize("Hq,Hk,D,past,new,window,prefix,mods", [
    (4, 2, 64, [500], [20], 40, 0, {}),
    (4, 2, 64, [500], [20], 40, 20, {}),
    (7, 1, 128, [500, 90, 1003], [20, 3, 1], 40, 0, {"cap": 20.0}),
    (8, 2, 128, [700, 0, 330], [300, 200, 77], 100, 37, {"bias": True}),      # several items a request, whose rows' windows begin at different keys
    (8, 2, 128, [20000], [5], 3000, 50, {}),                                    # cut into parts
    (8, 8, 64, [20000, 555], [1, 1], 1, 0, {"cap": 9.0, "bias": True}),
    (32, 8, 128, [4100], [900], 257, 128, {}),
], ids=str)
@pytest.mark.parametrize("entry", [-1, 1 << 28])
def test_released_blocks_do_not_matter(Hq, Hk, D, past, new, window, prefix, mods, entry):
    b = Batch(Hq, Hk, D, past, new, seed=41)
    more = {"cap": mods.get("cap", 0.0), "window": window, "slopes": slopes_of(Hq) if "bias" in mods else None,
            "prefix_lens": torch.full((len(past),), prefix, dtype=torch.int32, device=DEV) if prefix else None}
    prefill = lambda: b.pool.attn_prefill_chunk_scored(0, b.q, b.tables, b.cu, b.cu_host, b.seq_lens, b.scale, **more)
    last = (b.cu[1:] - 1).long()
    decode = lambda: b.pool.attn_decode_scored(0, b.q[last], b.tables, b.seq_lens, b.scale, **more)
    want, want_last = prefill(), decode()
    check(want, b.model(cap=more["cap"], window=window, slopes=more["slopes"], prefix=[prefix] * len(past) if prefix else None))
    blocks = list(gone(b, window, prefix))
    assert blocks
    for r, block in blocks:
        b.tables[r, block] = entry
    got, got_last = prefill(), decode()
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(got_last, want_last)
    assert b.pool.poll_status() == ekv.Status.OK
    seen = (b.past[0] - 1) // 16                                                # one that is looked at still counts
    if window > 1:
        b.tables[0, seen] = entry
        prefill()
        torch.cuda.synchronize()
        assert b.pool.poll_status() == ekv.Status.ERR_BLOCK_OOB
