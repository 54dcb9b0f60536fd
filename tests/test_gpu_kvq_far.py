"""The longest head that a table takes: byte offsets beyond 2^31, more rows than 24 bits count less one."""
import math

import pytest
import torch

import kvq_util as U
from paper_2601_13684_amd import binding as hc

pytestmark = pytest.mark.gpu
D, CAP = 128, 1 << 24


@pytest.mark.parametrize("n", [CAP, CAP - 33])
def test_rows_at_the_far_end(n):
    """Rows of zeros but for a few, whose sums are plain numbers: a weight of 1 to every zero row."""
    G = 4
    ctx = U.context(1, 1, G, CAP)
    cache = U.Cache(ctx, [CAP], gap=0)
    cache.arena.zero_()
    cache.acc.zero_()
    cache.state.copy_(torch.tensor([[n - 65, n - 65]], dtype=torch.int32))
    kv = torch.zeros((2 * n * D,), dtype=torch.bfloat16, device=U.DEV)
    x = torch.zeros((65, D), device=U.DEV)
    x[64], x[3] = 2.0, 1.0
    kv[(n - 65) * D:n * D] = x.to(torch.bfloat16).view(-1)
    kv[(2 * n - 65) * D:2 * n * D] = (3 * x).to(torch.bfloat16).view(-1)
    hc.hc_kvq_store(ctx, cache.kvq, kv, [0], [n * D], [n - 65], [65], cache.arena, cache.state, cache.acc)
    del kv
    assert cache.state.tolist() == [[n, n]]
    back = torch.zeros((2 * 70 * D,), dtype=torch.bfloat16, device=U.DEV)
    hc.hc_kvq_load(ctx, cache.kvq, cache.arena, cache.state, [n - 70], [70], back, [0], [70 * D])
    assert torch.equal(back[5 * D:70 * D].float().view(-1, D), x) and torch.equal(back[75 * D:].float().view(-1, D), 3 * x) and (back[:5 * D] == 0).all()
    q = torch.full((G, D), 1.0, device=U.DEV)
    q[1], q[2] = 0.5, 0.0
    out, lse = torch.zeros((G, D), device=U.DEV), torch.zeros((G,), device=U.DEV)
    work = cache.work()
    hc.hc_kvq_attn(ctx, cache.kvq, cache.arena, cache.state, q.to(torch.bfloat16), out, lse, cache.acc, 1.0, work, work.numel())
    weight = torch.zeros((2,), dtype=torch.float64)
    for g in range(G):
        s = [float(q[g, 0]) * D / math.sqrt(D) * k for k in (1.0, 2.0)]
        total = (n - 2) + math.exp(s[0]) + math.exp(s[1])
        p = torch.tensor([math.exp(s[0]) / total, math.exp(s[1]) / total], dtype=torch.float64)
        weight += p / G
        # (2^24 ones in parallel sums of at most 2^24 / 16384 terms: 2^-14; exponentials 2^-22 and the logits' roundings, here 2^-19)
        assert abs(float(out[g].double().mean()) / float(3 * p[0] + 6 * p[1]) - 1) <= 2.0 ** -13 and abs(float(lse[g]) - math.log(total)) <= 2.0 ** -13
        assert (out[g] == out[g, 0]).all()
    got = cache.acc[:n].double()
    assert abs(float(got[n - 65 + 3] / weight[0]) - 1) <= 2.0 ** -13 and abs(float(got[n - 1] / weight[1]) - 1) <= 2.0 ** -13
    assert abs(float(got.sum()) - 1) <= 2.0 ** -13 and float(got[:n - 65].max()) == float(got[:n - 65].min())
    # ---- the rows with the most weight
    to = U.Cache(ctx, [128], budget=[100], sink=10, recent=1)
    kept = torch.zeros((to.rows,), dtype=torch.int32, device=U.DEV)
    cache.acc[n // 2:n // 2 + 7] = 1.0
    hc.hc_kvq_evict(ctx, cache.kvq, cache.arena, cache.state, cache.acc, to.kvq, to.arena, to.state, to.acc, kept, work, work.numel())
    r = to.heads[0].row_off
    assert kept[r:r + 100].tolist() == list(range(91)) + list(range(n // 2, n // 2 + 7)) + [n - 65 + 3, n - 1]
    assert to.state.tolist() == [[100, n]]
    assert torch.equal(to.held(0, 0, 100)[98:], x[[3, 64]].double()) and torch.equal(to.held(0, 1, 100)[98:], 3 * x[[3, 64]].double())
    cache.close()
    to.close()
    hc.hc_destroy(ctx)
