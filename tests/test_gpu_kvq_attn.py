"""Attention over the cache held in 4 bits, and the rows' accumulated weights."""
import math

import pytest
import torch

import kvq_util as U
from paper_2601_13684_amd import binding as hc

pytestmark = pytest.mark.gpu
D = 128


def filled(ctx, rows, Hkv, seed=1, slack=40, kind="plain", spread=1.0):
    caps = [(n + slack + 15) // 16 * 16 for n in rows]
    cache = U.Cache(ctx, caps, rows=rows)
    for i, n in enumerate(rows):
        for v in (0, 1):
            if n:
                cache.put(i, v, 0, (U.rows_of(n, seed + 2 * i + v, kind).float() * (1.0 if v else spread)).to(torch.bfloat16))
    g = torch.Generator(device=U.DEV)
    g.manual_seed(seed)
    cache.acc = torch.rand((cache.rows,), generator=g, device=U.DEV) ** 4
    return cache


def run(ctx, cache, q, G, acc=True, decay=0.9):
    heads = len(cache.caps)
    out = torch.full((heads * G, D), 9.0, device=U.DEV)
    lse = torch.full((heads * G,), 9.0, device=U.DEV)
    work = cache.work()
    work.fill_(0xff)                                     # (NaNs: nothing may be read that the call has not written)
    before = cache.acc.clone()
    hc.hc_kvq_attn(ctx, cache.kvq, cache.arena, cache.state, q, out, lse, cache.acc if acc else None, decay, work, work.numel())
    return out, lse, before


def queries(heads, G, seed, scale=1.5):
    g = torch.Generator(device=U.DEV)
    g.manual_seed(seed)
    return (scale * torch.randn((heads * G, D), generator=g, device=U.DEV) + 0.3).to(torch.bfloat16)


@pytest.mark.parametrize("slack", [40, 2000])            # (tables of few rows a head are done in one launch)
@pytest.mark.parametrize("G", [1, 2, 4, 8])
@pytest.mark.parametrize("rows", [
    [1024], [1023, 993, 0, 512],
    [1], [31], [32], [33], [0, 0], [0, 5, 0], [127, 128, 129, 4097], [1000, 1, 0, 64, 31, 5000, 7, 0], [20011], [3] * 70, [0] * 66 + [100] + [0] * 10 + [70]])
def test_lengths(G, rows, slack):
    ctx = U.context(1, len(rows), G, max(rows) + 2100)
    cache = filled(ctx, rows, len(rows), slack=min(slack, 1024 - max(rows)) if slack == 40 and max(rows) <= 1024 else slack)
    q = queries(len(rows), G, 5)
    arena, state = cache.arena.clone(), cache.state.clone()
    out, lse, before = run(ctx, cache, q, G)
    U.check_attention(cache, q, G, out, lse, cache.acc, before, 0.9, (G, rows))
    untouched = torch.ones((cache.rows,), dtype=torch.bool, device=U.DEV)
    for h, n in zip(cache.heads, rows):
        untouched[h.row_off:h.row_off + n] = False
    assert torch.equal(cache.acc[untouched], before[untouched])
    assert torch.equal(cache.arena, arena) and torch.equal(cache.state, state)
    again = cache.acc.clone()                            # without weights: the same output, nothing accumulated
    out2, lse2, _ = run(ctx, cache, q, G, acc=False)
    assert torch.equal(out2, out) and torch.equal(lse2, lse) and torch.equal(cache.acc, again)
    cache.close()
    hc.hc_destroy(ctx)


@pytest.mark.parametrize("B,Hkv,G", [(1, 1, 8), (3, 2, 4), (16, 4, 2)])
def test_long_and_batched(B, Hkv, G):
    g = torch.Generator()
    g.manual_seed(B)
    rows = [int(math.exp(float(torch.rand((), generator=g)) * math.log(200000 / (B * Hkv)))) for _ in range(B * Hkv)]
    rows[0] = 300000 // (B * Hkv)
    ctx = U.context(B, Hkv, G, max(rows) + 100)
    cache = filled(ctx, rows, Hkv, seed=9)
    q = queries(B * Hkv, G, 6)
    out, lse, before = run(ctx, cache, q, G, decay=1.0)
    U.check_attention(cache, q, G, out, lse, cache.acc, before, 1.0, (B, Hkv, G))
    cache.close()
    hc.hc_destroy(ctx)


@pytest.mark.parametrize("slack", [40, 2000])
@pytest.mark.parametrize("G", [1, 4, 8])
def test_logits_far_apart(G, slack):
    """Logits of some thousand, rising along the rows, so that the reference moves all the time; the weights' differences are as exact as the logits."""
    n = 700
    ctx = U.context(1, 2, G, 2800)
    cache = filled(ctx, [n, n], 2, seed=4, spread=30.0, slack=slack)
    x = torch.ones((n, D), device=U.DEV) * torch.linspace(0.1, 40, n, device=U.DEV)[:, None]
    cache.put(1, 0, 0, x.to(torch.bfloat16))
    q = queries(2, G, 7, scale=6.0)
    out, lse, before = run(ctx, cache, q, G)
    U.check_attention(cache, q, G, out, lse, cache.acc, before, 0.9, G)
    cache.close()
    hc.hc_destroy(ctx)


@pytest.mark.parametrize("slack", [40, 2000])
@pytest.mark.parametrize("G", [1, 4, 8])
def test_values_of_any_size(G, slack):
    """Rows of values from 2^-120 to 2^70 under weights from 1 to 2^-60: every column is held to its own sum."""
    n = 300
    ctx = U.context(1, 1, G, 2400)
    cache = filled(ctx, [n], 1, seed=4, slack=slack)
    e = torch.randint(-120, 70, (n, 4), generator=torch.Generator().manual_seed(1)).to(U.DEV).double().repeat_interleave(32, dim=1)
    cache.put(0, 1, 0, (U.rows_of(n, 8).double() * 2.0 ** e).to(torch.bfloat16))
    q = queries(1, G, 7, scale=3.0)
    out, lse, before = run(ctx, cache, q, G)
    U.check_attention(cache, q, G, out, lse, cache.acc, before, 0.9, G)
    cache.close()
    hc.hc_destroy(ctx)


@pytest.mark.parametrize("slack", [40, 2000])
@pytest.mark.parametrize("G", [1, 4, 8])
def test_what_is_not_finite(G, slack):
    """NaNs behind the last row, in every byte, reach nothing.  A group of V that is not finite reaches its 32 columns of every query of its head and no others; a
    group of K every query of its head, and no other head."""
    rows = [70, 33, 200, 5]
    ctx = U.context(1, 4, G, 2300)
    cache = filled(ctx, rows, 4, slack=slack)
    for i, n in enumerate(rows):
        for v in (0, 1):
            codes, scales = cache.blocks(i, v)
            codes[n:], scales[n:] = 0, 255
    q = queries(4, G, 5)
    out, lse, before = run(ctx, cache, q, G)
    U.check_attention(cache, q, G, out, lse, cache.acc, before, 0.9, G)
    good = out.clone()
    cache.acc.copy_(before)
    cache.blocks(0, 1)[1][11, 2] = 255
    cache.blocks(2, 0)[1][150, 1] = 255
    out, lse, _ = run(ctx, cache, q, G)
    bad = torch.zeros_like(out, dtype=torch.bool)
    bad[:G, 64:96] = True
    bad[2 * G:3 * G] = True
    assert torch.equal(out.isnan(), bad) and torch.equal(out[~bad], good[~bad])
    assert torch.equal(lse.isnan(), torch.arange(4 * G, device=U.DEV) // G == 2)
    r = [cache.heads[i].row_off for i in range(4)]
    assert cache.acc[r[2]:r[2] + 200].isnan().all() and not cache.acc[r[0]:r[0] + 70].isnan().any()
    cache.close()
    hc.hc_destroy(ctx)


def test_same_bits_every_time_and_states_out_of_range():
    rows = [5000, 300, 0, 77]
    ctx = U.context(2, 2, 4, 6000)
    cache = filled(ctx, rows, 2)
    q = queries(4, 4, 5)
    start = cache.acc.clone()
    out, lse, _ = run(ctx, cache, q, 4)
    first = cache.acc.clone()
    for _ in range(3):
        cache.acc.copy_(start)
        out2, lse2, _ = run(ctx, cache, q, 4)
        assert torch.equal(out, out2) and torch.equal(lse, lse2) and torch.equal(first, cache.acc)
    for i in range(4):                                   # rows of the whole room: what a length beyond it is taken as
        for v in (0, 1):
            codes, scales = cache.blocks(i, v)
            codes[rows[i]:], scales[rows[i]:] = 0x31, 126
    cache.state[:, 0] = torch.tensor([1 << 30, 300, -5, 77], dtype=torch.int32)
    out, lse, before = run(ctx, cache, q, 4)
    cache.state[:, 0] = torch.tensor([cache.caps[0], 300, 0, 77], dtype=torch.int32)
    U.check_attention(cache, q, 4, out, lse, cache.acc, before, 0.9)
    cache.close()
    hc.hc_destroy(ctx)
