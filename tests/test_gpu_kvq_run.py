"""The operators of the cache held in 4 bits one after the other, as a program uses them: prompt, decode tokens, eviction, captured steps, other streams."""
import math

import pytest
import torch

import kvq_util as U
from paper_2601_13684_amd import binding as hc
from paper_2601_13684_amd import runtime as R

pytestmark = pytest.mark.gpu
DEV, D = U.DEV, U.D


def context(B, Hkv, G, max_ctx):
    return R.Context(hc.hc_config(B=B, Hq=Hkv * G, Hkv=Hkv, D=D, max_ctx=(max_ctx + 63) // 64 * 64, max_k=8, window=1, metric=0, tau_num=1, tau_den=2, agg=0,
                                  window_mode=0), DEV)


def tokens(n, Hq, Hkv, seed, dtype=torch.bfloat16):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    x = (torch.randn((n, Hq + 2 * Hkv, D), generator=g, device=DEV) * torch.exp(0.3 * torch.randn((Hq + 2 * Hkv, D), generator=g, device=DEV))).to(dtype)
    return x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]


class View:
    """What check_attention looks at, of a QuantCache."""

    def __init__(self, c):
        self.caps, self.heads, self.state, self.arena = c.table.room, c.table.heads, c.state, c.arena

    blocks, held = U.Cache.blocks, U.Cache.held


def values(c, i):
    """Rows that head i holds, K and V."""
    n = c.rows()[i]
    v = View(c)
    return [v.held(i, side, n) for side in (0, 1)]


@pytest.mark.parametrize("G,layout,dtype", [(4, hc.HC_ROPE_HALF, torch.bfloat16), (8, hc.HC_ROPE_INTERLEAVED, torch.float32), (1, hc.HC_ROPE_HALF, torch.bfloat16)])
def test_prompt_tokens_eviction_tokens(G, layout, dtype):
    print("kvq run", G, layout, dtype, flush=True)
    B, Hkv, lens, steps = 2, 2, [700, 1023], 4
    Hq = Hkv * G
    ctx = context(B, Hkv, G, 1200)
    w = [1 + 0.1 * torch.randn((D,), device=DEV) for _ in range(2)]
    rope = hc.hc_rope_init(layout, 128, 10000.0, q_norm=w[0], k_norm=w[1])
    prompt = R.Prompt(ctx, lens)
    room = [n + 20 for n in lens for _ in range(Hkv)]
    cache = R.QuantCache(R.QuantTable(ctx, room))
    for count in ([1, 500], [400, 0], [299, 523]):
        first = list(prompt.length)
        prompt.chunk(rope, *tokens(sum(count), Hq, Hkv, sum(first) + 1, dtype), count)
        cache.store(prompt, first, count)
    assert cache.rows() == [n for n in lens for _ in range(Hkv)]
    for i in range(B * Hkv):
        for side, off in ((0, prompt.k_off[i]), (1, prompt.v_off[i])):
            rows = prompt.kv[off:off + lens[i // Hkv] * D].view(-1, D)
            assert torch.equal(values(cache, i)[side], U.decode(*U.encode(rows))), (i, side)

    def step(cache, seed, decay):
        q = cache.append_rope(rope, *tokens(B, Hq, Hkv, seed, dtype))
        before = cache.acc.clone()
        out, lse = cache.attn(q, decay)
        U.check_attention(View(cache), q, G, out, lse, cache.acc, before, decay, seed)
        return out, lse
    for t in range(steps):
        step(cache, 100 + t, 0.95)
    # ---- to budgets, and on
    budget = [150, 333, 1027, 40]
    small = R.QuantCache(R.QuantTable(ctx, [b + 16 for b in budget], budget, sink=4, recent=20))
    for turn in range(2):                                # (the second time into the first cache's place)
        kept = torch.full((small.table.rows,), -1, dtype=torch.int32, device=DEV)
        held = [values(cache, i) for i in range(B * Hkv)]
        rows, acc, pos = cache.rows(), cache.acc.clone(), cache.state[:, 1].clone()
        cache.evict(small, kept)
        for i in range(B * Hkv):
            a, b = cache.table.heads[i].row_off, small.table.heads[i].row_off
            stay = U.survivors(rows[i], budget[i], 4, 20, acc[a:a + rows[i]])
            at = torch.tensor(stay, device=DEV)
            assert kept[b:b + len(stay)].tolist() == stay
            for side in (0, 1):
                assert torch.equal(values(small, i)[side], held[i][side][at])
            assert torch.equal(small.acc[b:b + len(stay)], acc[a + at])
        assert torch.equal(small.state[:, 1], pos)
        for t in range(steps):
            step(small, 200 + 10 * turn + t, 1.0)
        if turn == 0:
            again = R.QuantCache(R.QuantTable(ctx, [b + 32 for b in budget], budget, sink=4, recent=20), work=cache.work)
            cache, small = small, again
    torch.cuda.synchronize()
    ctx.close()


def test_attention_agrees_with_the_bf16_path():
    """hc_decode_attn over the rows that hc_kvq_load gives back."""
    B, Hkv, G, n = 1, 2, 4, 5000
    ctx = context(B, Hkv, G, n + 64)
    prompt = R.Prompt(ctx, [n])
    rope = hc.hc_rope_init(hc.HC_ROPE_HALF, 128, 10000.0)
    q, _, _ = prompt.chunk(rope, *tokens(n, Hkv * G, Hkv, 3), [n])
    cache = R.QuantCache(R.QuantTable(ctx, [n] * Hkv), weights=False)
    cache.store(prompt, [0], [n])
    back = torch.zeros_like(prompt.kv)
    cache.load([0], [n], back, prompt.k_off, prompt.v_off)
    descs = (hc.hc_head_desc * Hkv)(*[hc.hc_head_desc(k_off=prompt.k_off[h], v_off=prompt.v_off[h], tier_off=0, ctx=n, len=n, role=0, rep=-1) for h in range(Hkv)])
    layer = hc.hc_layer_create(ctx.handle, list(descs))
    want, want_lse = torch.empty((1, Hkv * G, D), device=DEV), torch.empty((1, Hkv * G), device=DEV)
    last = q[-1:].contiguous()
    hc.hc_decode_attn(ctx.handle, layer, back, last, want, want_lse)
    out, lse = cache.attn(last)
    # (both are 32-bit; a logit is off by 2^-24 (130 sum |q k| / sqrt(128) + 4 |s|) at most, see check_attention: here below 2^-12, in either, twice in a ratio)
    scale = back.float().abs().max()
    assert (out - want).abs().max() <= 2.0 ** -10 * scale and (lse - want_lse).abs().max() <= 1e-4
    torch.cuda.synchronize()
    hc.hc_layer_destroy(layer)
    ctx.close()


def test_a_captured_step():
    """Append and attention in a graph, replayed while the lengths grow, beside an eager cache that takes the same tokens, and an eviction in a graph of its own."""
    B, Hkv, G, steps = 3, 2, 4, 40
    Hq = Hkv * G
    ctx = context(B, Hkv, G, 300)
    rope = hc.hc_rope_init(hc.HC_ROPE_HALF, 128, 10000.0)
    table = R.QuantTable(ctx, [16, 32, 48, 64, 80, 96])
    to = R.QuantTable(ctx, [16] * 6, [8, 8, 9, 10, 11, 16], 1, 2)
    a, b = R.QuantCache(table), R.QuantCache(table)
    ta, tb = R.QuantCache(to), R.QuantCache(to)
    x = torch.zeros((B, Hq + 2 * Hkv, D), dtype=torch.bfloat16, device=DEV)
    q, out, lse = (torch.empty(s, dtype=t, device=DEV) for s, t in (((B, Hq, D), torch.bfloat16), ((B, Hq, D), torch.float32), ((B, Hq), torch.float32)))
    parts = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]

    def step(c, q, out, lse):
        c.append_rope(rope, *parts, q)
        c.attn(q, 0.9, out, lse)
    q2, out2, lse2 = torch.empty_like(q), torch.empty_like(out), torch.empty_like(lse)
    torch.cuda.synchronize()
    graph, gone = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(a, q, out, lse)
    with torch.cuda.graph(gone):
        a.evict(ta)
    g = torch.Generator(device=DEV)
    g.manual_seed(5)
    for t in range(steps):
        x.copy_(torch.randn(x.shape, generator=g, device=DEV).to(torch.bfloat16))
        graph.replay()
        step(b, q2, out2, lse2)
        if t % 9 == 4:
            gone.replay()
            b.evict(tb)
            torch.cuda.synchronize()
            for k in ("arena", "state", "acc"):
                assert torch.equal(getattr(ta, k), getattr(tb, k)), (t, k)
        assert torch.equal(out, out2) and torch.equal(lse, lse2) and torch.equal(q, q2), t
        assert torch.equal(a.state, b.state) and torch.equal(a.acc, b.acc) and torch.equal(a.arena, b.arena), t
    assert a.rows() == [16, 32, 40, 40, 40, 40] and a.state[:, 1].tolist() == [steps] * 6
    del graph, gone
    torch.cuda.synchronize()
    ctx.close()


def test_made_and_dropped_while_the_other_stream_works():
    """The current stream is busy when the buffers are made, the side stream does not wait for it by itself, and the caches are gone, their memory asked for
    and overwritten, before either is through."""
    B, Hkv, G, n = 1, 2, 4, 3000
    Hq = Hkv * G
    ctx = context(B, Hkv, G, n + 64)
    rope = hc.hc_rope_init(hc.HC_ROPE_HALF, 64, 10000.0)
    table, to = R.QuantTable(ctx, [n + 16] * Hkv), R.QuantTable(ctx, [512] * Hkv, [500] * Hkv, 4, 50)
    prompt = R.Prompt(ctx, [n])
    prompt.chunk(rope, *tokens(n, Hq, Hkv, 3), [n])
    new = tokens(B, Hq, Hkv, 4)

    def work(stream):
        cache, small = R.QuantCache(table), R.QuantCache(to)
        cache.store(prompt, [0], [n], stream)
        q = cache.append_rope(rope, *new, stream=stream)
        out, lse = cache.attn(q, 1.0, stream=stream)
        cache.evict(small, stream=stream)
        with torch.cuda.stream(stream):
            got = [t.clone() for t in (out, lse, small.state, small.acc, small.arena)]
        return got, [cache.arena.numel(), cache.work.numel(), small.arena.numel()]
    want, sizes = work(torch.cuda.current_stream())
    side, busy = torch.cuda.Stream(), torch.empty((1 << 28,), dtype=torch.float32, device=DEV)
    for _ in range(3):
        torch.cuda.synchronize()
        for _ in range(40):
            busy.fill_(1.0)                      # milliseconds of work in front of the buffers' fill
        got, _ = work(side)
        noise = [torch.full((s,), 255, dtype=torch.uint8, device=DEV) for s in sizes]
        side.synchronize()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want))
        del noise
    ctx.close()


def test_refused():
    ctx = context(1, 2, 4, 128)
    table = R.QuantTable(ctx, [20, 40])
    assert table.room == [32, 48]
    a, b = R.QuantCache(table, weights=False), R.QuantCache(table)
    with pytest.raises(ValueError):
        R.QuantTable(ctx, [64])
    with pytest.raises(ValueError):
        R.QuantTable(ctx, [64, 64], [1])
    with pytest.raises(hc.HcError):
        R.QuantTable(ctx, [64, 256])
    with pytest.raises(ValueError):
        a.evict(b)
    with pytest.raises(hc.HcError):
        b.evict(b)
    prompt = R.Prompt(ctx, [64])
    with pytest.raises(ValueError):
        a.store(prompt, [0], [1])
    q = torch.zeros((1, 8, D), dtype=torch.bfloat16, device=DEV)
    with pytest.raises(ValueError):
        a.attn(q[:, :4].contiguous())
    with pytest.raises(ValueError):
        a.attn(q.float())
    with pytest.raises(ValueError):
        a.attn(q, out=torch.zeros((1, 8, 64), device=DEV))
    with pytest.raises(hc.HcError):
        b.attn(q, decay=math.nan)
    torch.cuda.synchronize()
    ctx.close()
