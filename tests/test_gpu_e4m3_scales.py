"""V scales of one sequence very far apart: what the formats of P keep, as include/ekv.h states it."""
import math

import numpy as np
import pytest
import torch

import e4m3_model as M
import ekv_inputs as I
import paper_2608_23658_b200 as ekv
from test_gpu_e4m3 import Case, DEV

pytestmark = pytest.mark.gpu


def spread_out(c, up, zero_channels):
    """Every third block's V scale up by 2^up, its codes 0 in some channels; K and V of the case as they are stored then."""
    ids = torch.cat([c.tables[b, :-(-L // 16):3] for b, L in enumerate(c.lengths)]).long().to(DEV)
    c.pool.layer_scales(0)[ids, 1] *= 2.0 ** up
    codes = c.pool.layer_tensor(0).view(torch.uint8)
    v = codes[ids, 1]
    v[..., zero_channels] = 0
    codes[ids, 1] = v
    kk, vv = (x.double().cpu() for x in c.pool.read_kv(0, torch.cat(c.slots).to(DEV)))
    c.K, c.V = list(kk.split(c.lengths)), list(vv.split(c.lengths))


@pytest.mark.parametrize("shape", [I.LLAMA8B, I.Shape(8, 2, 64)], ids=str)
@pytest.mark.parametrize("up", [12, 45, 90])
def test_channels_that_the_largest_scales_have_zeros_in(shape, up):
    """Decode and few rows hold to the bound with its absolute part, 2^-31 of the largest weight times scale a key; the kernel for
    many rows multiplies the scale into V and needs none, so in those channels it sees what the blocks of small scale hold."""
    c = Case(shape, [700, 333], seed=up)
    with c.pool:
        zero = torch.arange(0, shape.head_dim, 3)
        spread_out(c, up, zero)
        scale = 0.5 / math.sqrt(shape.head_dim)
        q = c.queries(2)
        c.check_decode(q, c.pool.attn_decode(0, q.to(DEV), c.d_tables, c.d_lens, scale), scale, f"2^{up}")
        for chunks, bare in (([5, 2], False), ([150, 333], True)):
            cu = torch.tensor(np.concatenate([[0], np.cumsum(chunks)]), dtype=torch.int32)
            q = c.queries(int(cu[-1]))
            out = c.pool.attn_prefill_chunk(0, q.to(DEV), c.d_tables, cu.to(DEV), cu, c.d_lens, scale)
            for r, (n, L) in enumerate(zip(chunks, c.lengths)):
                a, b = int(cu[r]), int(cu[r + 1])
                want, bound = M.attention(q[a:b].double(), c.K[r], c.V[r], torch.arange(L - n, L) + 1, scale, None if bare else c.sv(r))
                M.assert_within(out[a:b], want, bound, f"{chunks[r]} rows of {L}, 2^{up}")
                if bare:
                    assert (want[..., zero].abs() > 8 * bound[..., zero]).float().mean() > 0.5  # the bound says something there
        assert c.pool.poll_status() == ekv.Status.OK
