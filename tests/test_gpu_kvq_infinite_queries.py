"""Queries that are not finite, over the cache held in 4 bits.  Run with `-m gpu` on an MI355X."""
import math

import pytest
import torch

import kvq_util as U
from paper_2601_13684_amd import binding as hc

pytestmark = pytest.mark.gpu
D = 128


@pytest.mark.parametrize("caps", [[128, 64, 64], [2048, 1040, 1040]])
@pytest.mark.parametrize("G", [1, 2, 4, 8])
@pytest.mark.parametrize("bad", [-math.inf, math.inf, math.nan])
def test_a_query_that_is_not_finite(caps, G, bad):
    """Element 9 of a query of head 0 and of the head without rows: with positive keys there, every logit is the same infinity.  The outputs are no numbers, as a softmax of such
    is none; the head's other queries, and other heads, are what they were, and so is a head without rows."""
    rows = [100, 0, 40]
    ctx = U.context(1, 3, G, 2048)
    cache = U.Cache(ctx, caps, rows=rows)
    for i, n in enumerate(rows):
        for v in (0, 1):
            if n:
                x = U.rows_of(n, 3 + 2 * i + v)
                x[:, 9] = 1.0 + x[:, 9].abs().clamp(max=1.0)
                cache.put(i, v, 0, x)
    q = torch.randn((3 * G, D), generator=torch.Generator(device=U.DEV).manual_seed(1), device=U.DEV).to(torch.bfloat16)

    def run(q):
        cache.acc.fill_(0.25)
        out, lse = torch.full((3, G, D), 9.0, device=U.DEV), torch.full((3, G), 9.0, device=U.DEV)
        work = cache.work()
        hc.hc_kvq_attn(ctx, cache.kvq, cache.arena, cache.state, q, out, lse, cache.acc, 1.0, work, work.numel())
        torch.cuda.synchronize()
        return out, lse, cache.acc.clone()
    good = run(q)
    q[G - 1, 9], q[G, 9] = bad, bad
    out, lse, acc = run(q)
    assert out[0, G - 1].isnan().all() and (lse[0, G - 1] == bad or lse[0, G - 1].isnan())
    assert torch.equal(out[0, :G - 1], good[0][0, :G - 1]) and torch.equal(lse[0, :G - 1], good[1][0, :G - 1])
    assert (out[1] == 0).all() and (lse[1] == -math.inf).all()
    assert torch.equal(out[2], good[0][2]) and torch.equal(lse[2], good[1][2])
    r = [h.row_off for h in cache.heads]
    assert acc[r[0]:r[0] + 100].isnan().all()
    acc[r[0]:r[0] + 100] = good[2][r[0]:r[0] + 100]
    assert torch.equal(acc, good[2])
    cache.close()
    hc.hc_destroy(ctx)
