"""Which shared calls read the shared keys once and which read every request's: the other tests' groups are meant to stand on both sides of that rule."""
import pytest
import torch

import paper_2608_23658_b200 as ekv
from scored_model import check
from test_gpu_decode_shared import make, run

pytestmark = pytest.mark.gpu


def reads_once(b):
    """A call that reads shared keys once cuts its own keys and keeps parts of the shared ones; one that does not needs what the same batch does
    without shared keys."""
    need = lambda shared: ekv.ekv_attn_decode_shared_workspace_bytes(b.pool.handle, b.starts, shared, b.tables.shape[1])
    return need(b.shared) != need(torch.zeros_like(b.shared))


SMALL, LARGE = [(4, 2, 64), (5, 1, 64)], [(28, 4, 128), (8, 8, 64), (6, 2, 128), (64, 8, 128)]


@pytest.mark.parametrize("Hq,Hk,D", SMALL + LARGE)
@pytest.mark.parametrize("groups,own", [([(2, 16)], [1, 40]), ([(4, 512)], [1, 17, 40, 16]), ([(2, 12000)], [1, 40]), ([(2, 1024)], [500, 900]),
                                        ([(2, 16), (4, 64), (2, 12000), (3, 128), (1, 48), (0, 0), (5, 0)], [3, 100, 15, 1])], ids=str)
def test_small_groups_read_their_keys_themselves(Hq, Hk, D, groups, own):
    b = make(Hq, Hk, D, groups, own, seed=71)
    assert not reads_once(b)
    check(run(b), b.model())


@pytest.mark.parametrize("Hq,Hk,D", SMALL + LARGE)
@pytest.mark.parametrize("groups,own", [([(2, 36000)], [1, 40]), ([(6, 36000), (3, 0)], [30]), ([(40, 11904), (3, 2000)], [1, 9, 33]),
                                        ([(37, 1040), (70, 12016), (33, 48)], [20, 64])], ids=str)
def test_large_groups_and_long_prefixes_are_read_once(Hq, Hk, D, groups, own):
    b = make(Hq, Hk, D, groups, own, seed=72)
    assert reads_once(b)
    check(run(b), b.model())


@pytest.mark.parametrize("Hq,Hk,D", [(28, 4, 128), (8, 8, 64), (64, 8, 128)])
def test_prefixes_of_12000_are_read_once_for_six_requests_of_many_heads(Hq, Hk, D):
    b = make(Hq, Hk, D, [(6, 12000), (2, 32)], [16, 3], seed=73)
    assert reads_once(b)
    b.seq_lens[1], b.seq_lens[4] = 12000, 12000                       # no keys of their own
    b.lens[1], b.lens[4] = 12000, 12000
    b.seq_lens[2] = b.lens[2] = 0                                     # padding
    got, (want, bound) = run(b), b.model()
    assert (got[2] == 0).all()
    check(got, (want, bound))
    b.cache[int(b.tables[3, 750]), 1, 0, 2, 9] = float("nan")         # an own value of request 3
    hurt = run(b)
    group = Hq // Hk
    assert torch.isnan(hurt[3, :group, 9]).all()
    hurt[3, :group, 9] = got[3, :group, 9]
    assert torch.equal(hurt, got) and b.pool.poll_status() == ekv.Status.OK
    b.tables[0, 7] = -5                                               # a shared block
    assert torch.isfinite(run(b)[[0, 1, 4, 5]]).all()
    torch.cuda.synchronize()
    assert b.pool.poll_status() == ekv.Status.ERR_BLOCK_OOB
