"""Calls of several threads on one stream share the pool's workspace of that stream: their launches may not fall between one another (no GPU needed)."""
import threading
import time

import pytest
import torch

import paper_2608_23658_b200 as ekv
from paper_2608_23658_b200 import _binding, pool as pool_module
from test_binding_checks import gpu
from test_scored_binding_checks import pool_of

BF16 = torch.bfloat16


@pytest.fixture
def library(monkeypatch):
    """A library whose calls take their time and count those that are inside at once."""
    class Lib:
        inside = most = 0
        seen = []

        def __getattr__(self, name):
            if name in ("ekv_last_error", "ekv_status_string"):
                return lambda *args: b"refused"

            def call(*args):
                Lib.inside += 1
                Lib.most = max(Lib.most, Lib.inside)
                Lib.seen.append((name, args))
                time.sleep(0.02)
                Lib.inside -= 1
                return 0
            return call

    monkeypatch.setattr(_binding, "load_library", lambda: Lib())
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(pool_module, "_raw_stream", lambda device: 7)
    return Lib


def test_calls_that_share_a_workspace_are_made_one_after_the_other(library):
    pool, R = pool_of(), 3
    pool._lock = threading.Lock()
    kept = torch.zeros(512, dtype=torch.uint8)
    pool._parts[7] = [kept]
    starts, shared, cu = torch.tensor([0, R], dtype=torch.int32), torch.tensor([32], dtype=torch.int32), torch.arange(R + 1, dtype=torch.int32)
    q, tables, lens = gpu(R, 4, 64, dtype=BF16), gpu(R, 9), gpu(R)
    outs = [gpu(R, 4, 64, dtype=BF16) for _ in range(6)]
    calls = [lambda out: pool.attn_decode_shared(0, q, tables, lens, starts, shared, 0.5, out=out),
             lambda out: pool.attn_decode_scored(0, q, tables, lens, 0.5, cap=3.0, out=out),
             lambda out: pool.attn_prefill_chunk_scored(0, q, tables, gpu(R + 1), cu, lens, 0.5, cap=3.0, out=out)]
    threads = [threading.Thread(target=calls[i % 3], args=(out,)) for i, out in enumerate(outs)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert len(library.seen) == 6 and all(kept.data_ptr() in args for _, args in library.seen)
    assert library.most == 1


def test_a_refused_call_leaves_the_pool_usable(library, monkeypatch):
    pool = pool_of()
    pool._lock = threading.Lock()
    pool._parts[7] = [torch.zeros(512, dtype=torch.uint8)]
    refuse = lambda *args: ekv.Status.ERR_INVALID
    with pytest.raises(ekv.EkvError):
        pool._launch(refuse, lambda: 1, None, None)
    assert pool._launch(lambda *args: 0, lambda: 1, None, None) is None
