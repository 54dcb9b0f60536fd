"""Eviction from the cache held in 4 bits by accumulated weight, and the operators of that cache one after the other."""
import math

import pytest
import torch

import kvq_util as U
from paper_2601_13684_amd import binding as hc

pytestmark = pytest.mark.gpu
D = 128


def weights(n, kind, g):
    x = torch.exp(2 * torch.randn((n,), generator=g, device=U.DEV))
    if kind == "ties":
        x = torch.randint(0, 4, (n,), generator=g, device=U.DEV).float()
    if kind == "zeros":
        x.zero_()
        x[::7] = -0.0
    if kind == "close":          # keys that differ in their last bits alone
        x = 1 + torch.randint(0, 3000, (n,), generator=g, device=U.DEV).float() * 2.0 ** -23
    if kind == "odd":
        x[torch.rand((n,), generator=g, device=U.DEV) < 0.3] = math.nan
        x[torch.rand((n,), generator=g, device=U.DEV) < 0.1] = math.inf
        x[torch.rand((n,), generator=g, device=U.DEV) < 0.1] = -math.inf
        x *= 1 - 2 * torch.randint(0, 2, (n,), generator=g, device=U.DEV)
    return x


@pytest.mark.parametrize("kind", ["plain", "ties", "zeros", "close", "odd"])
@pytest.mark.parametrize("B,Hkv,rows,budget,sink,recent,kept", [
    (1, 2, [300, 300], [100, 33], 4, 16, True), (1, 3, [1, 0, 64], [1, 5, 64], 0, 0, True), (2, 2, [2000, 1999, 5, 1023], [1998, 1, 4, 1022], 0, 1, False),
    (1, 1, [1500], [200], 128, 72, True), (1, 2, [40000, 37000], [30000, 129], 64, 64, True), (3, 1, [50000, 12, 36865], [49999, 100, 2000], 100, 0, False),
    (1, 2, [900, 900], [300, 900], 150, 100, True), (1, 1, [40], [64], 50, 50, True), (1, 2, [20000, 9000], [15000, 11000], 5000, 6000, True),
    (1, 2, [8193, 16385], [8192, 4096], 0, 0, False), (1, 2, [1, 28], [32, 48], 4, 4096, True), (1, 2, [9000, 40], [9100, 9000], 2 ** 30, 2 ** 30, True)])
def test_what_stays(kind, B, Hkv, rows, budget, sink, recent, kept):
    heads = B * Hkv
    ctx = U.context(B, Hkv, 2, max(rows) + 100)
    cache = U.Cache(ctx, [(n + 15) // 16 * 16 + 16 for n in rows], rows=rows, pos=[n + 1000 for n in rows])
    g = torch.Generator(device=U.DEV)
    g.manual_seed(7)
    cache.arena.copy_(torch.randint(0, 256, (cache.bytes,), generator=g, dtype=torch.uint8, device=U.DEV))
    cache.acc = weights(cache.rows, kind, g)
    to = U.Cache(ctx, [(b + 15) // 16 * 16 + 16 for b in budget], budget=budget, sink=sink, recent=recent)
    was = {k: getattr(to, k).clone() for k in ("arena", "acc")}
    source = {k: getattr(cache, k).clone() for k in ("arena", "acc", "state")}
    lst = torch.full((to.rows,), -7, dtype=torch.int32, device=U.DEV) if kept else None
    want_list = None if lst is None else lst.clone()
    work = cache.work()
    hc.hc_kvq_evict(ctx, cache.kvq, cache.arena, cache.state, cache.acc, to.kvq, to.arena, to.state, to.acc, lst, work, work.numel())
    for i in range(heads):
        h, t = cache.heads[i], to.heads[i]
        stay = U.survivors(rows[i], budget[i], sink, recent, cache.acc[h.row_off:h.row_off + rows[i]])
        m, at = len(stay), torch.tensor(stay, dtype=torch.int64, device=U.DEV)
        assert to.state[i].tolist() == [m, rows[i] + 1000], i
        was["acc"][t.row_off:t.row_off + m] = cache.acc[h.row_off + at]
        if kept:
            want_list[t.row_off:t.row_off + m] = at.int()
        for v in (0, 1):
            c, s = cache.blocks(i, v)
            off = t.off + 68 * t.cap * v
            was["arena"][off:off + 64 * m] = c[at].view(-1)
            was["arena"][off + 64 * t.cap:off + 64 * t.cap + 4 * m] = s[at].view(-1)
    if kept:
        assert torch.equal(lst, want_list)
    assert torch.equal(to.acc.view(torch.int32), was["acc"].view(torch.int32)) and torch.equal(to.arena, was["arena"])
    for k, x in source.items():
        assert torch.equal(getattr(cache, k).view(torch.uint8), x.view(torch.uint8)), k
    cache.close()
    to.close()
    hc.hc_destroy(ctx)
