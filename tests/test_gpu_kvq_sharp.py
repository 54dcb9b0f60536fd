"""Attention over the cache held in 4 bits, row for row: every row counts once, no weight loses a part.  Run with `-m gpu` on an MI355X."""
import math

import pytest
import torch

import kvq_sharp_util as S
import kvq_util as U
from paper_2601_13684_amd import binding as hc

pytestmark = pytest.mark.gpu
D = 128


def attend(ctx, cache, q, G, acc):
    heads = len(cache.caps)
    out, lse = torch.full((heads, G, D), 9.0, device=U.DEV), torch.full((heads, G), 9.0, device=U.DEV)
    work = cache.work()
    work.fill_(0xff)
    cache.acc.fill_(8.0)
    hc.hc_kvq_attn(ctx, cache.kvq, cache.arena, cache.state, q, out, lse, cache.acc if acc else None, 0.0, work, work.numel())
    torch.cuda.synchronize()
    return out, lse


def check(cache, out, lse, acc, one):
    """one(i, n, out, lse, weights): head i's check."""
    for i, n in enumerate(cache.state[:, 0].tolist()):
        if n == 0:
            assert (out[i] == 0).all() and (lse[i] == -math.inf).all(), i
            continue
        r = cache.heads[i].row_off
        one(i, n, out[i], lse[i], cache.acc[r:r + n] if acc else None)
        assert (cache.acc[r + (n if acc else 0):r + cache.caps[i]] == 8.0).all(), i


def every_row_once(rows, caps, G, acc, B=1, runs=S.RUNS):
    ctx = U.context(B, len(rows) // B, G, max(caps))
    cache = U.Cache(ctx, caps, rows=rows)
    q = torch.randn((len(rows) * G, D), generator=torch.Generator(device=U.DEV).manual_seed(3), device=U.DEV).to(torch.bfloat16)
    for run in runs:
        for i in range(len(rows)):
            S.put_ones(cache, i, run)
        out, lse = attend(ctx, cache, q, G, acc)
        check(cache, out, lse, acc, lambda i, n, o, l, w: S.check_ones(o, l, w, n, run, (i, run)))  # noqa: B023
    cache.close()
    hc.hc_destroy(ctx)


def nothing_lost(rows, caps, G, acc, B=1):
    ctx = U.context(B, len(rows) // B, G, max(caps))
    cache = U.Cache(ctx, caps, rows=rows)
    g = torch.Generator(device=U.DEV).manual_seed(5)
    for v in (0, 1):
        codes, scales = (x.split(rows) for x in U.encode(torch.randn((sum(rows), D), generator=g, device=U.DEV).to(torch.bfloat16)))
        for i, n in enumerate(rows):
            c, s = cache.blocks(i, v)
            c[:n], s[:n] = codes[i], scales[i]
    q = torch.randn((len(rows) * G, D), generator=g, device=U.DEV).to(torch.bfloat16)
    out, lse = attend(ctx, cache, q, G, acc)

    def one(i, n, o, l, w):
        K, V = cache.held(i, 0, n), cache.held(i, 1, n)
        if n >= 100:
            S.check_rms(o, l, w, q.view(-1, G, D)[i], K, V, i)
    check(cache, out, lse, acc, one)
    cache.close()
    hc.hc_destroy(ctx)


def up(n):
    return max(16, (n + 15) // 16 * 16)


ROWS = [([300, 1000, 31, 1], 1024), ([130, 512, 33, 0], 512), ([256, 100, 65, 16], 256), ([700, 1024, 0, 33], 4096), ([20011, 1, 0, 3000], 20016), ([150000, 77, 1024, 40000], 150016)]


@pytest.mark.parametrize("acc", [True, False])
@pytest.mark.parametrize("G", [1, 2, 4, 8])
@pytest.mark.parametrize("rows,most", ROWS)
@pytest.mark.parametrize("what", [every_row_once, nothing_lost])
def test_lengths(what, rows, most, G, acc):
    what(rows, [min(most, up(n + 50)) for n in rows[:3]] + [most], G, acc)


@pytest.mark.parametrize("G", [1, 4, 8])
def test_one_long_head(G):
    every_row_once([300000], [300000], G, True)
    nothing_lost([300000], [300000], G, True)


def drawn(n, most, seed):
    """n lengths up to most, some of them 0."""
    g = torch.Generator().manual_seed(seed)
    return [0 if float(torch.rand((), generator=g)) < 0.1 else int(most ** float(torch.rand((), generator=g))) for _ in range(n)]


@pytest.mark.parametrize("acc", [True, False])
@pytest.mark.parametrize("heads,G", [(768, 1), (772, 1), (192, 4), (196, 4), (96, 8), (100, 8), (1024, 1), (1028, 1), (256, 4), (260, 4), (128, 8), (132, 8)])
def test_many_query_heads(heads, G, acc):
    """On either side of what workgroups of either size join: heads of up to 1,500 rows, some without any."""
    rows = drawn(heads, 1500, heads)
    every_row_once(rows, [up(max(n, 1030 if i == 5 else 1)) for i, n in enumerate(rows)], G, acc, B=heads // 4, runs=(1, 32))
    nothing_lost(rows, [up(max(n, 1030 if i == 5 else 1)) for i, n in enumerate(rows)], G, acc, B=heads // 4)


@pytest.mark.parametrize("heads,G", [(520, 1), (600, 2), (1100, 1), (516, 8)])
@pytest.mark.parametrize("long", [0, 515])
def test_more_heads_than_a_wave_has_lanes_eight_times(heads, G, long):
    """Every lane looks through more than eight heads to find its workgroup's share; one head is long, the others a few rows."""
    rows = drawn(heads, 60, heads + long)
    rows[long] = 100001
    every_row_once(rows, [up(n + 1) for n in rows], G, True, B=heads // 4)


def table_of(ctx, caps, budget=None):
    return U.Cache(ctx, caps, rows=None, budget=budget, sink=4, recent=16)


def test_captured_over_long_heads():
    """Append and attention of long heads, replayed while heads come into new tiles and all of them into larger shares; the eviction of such heads in a graph of its own.  Beside
    an eager cache that takes the same tokens."""
    B, Hkv, G, steps = 4, 2, 4, 45
    Hq, caps = Hkv * G, [8224, 8240, 16400, 8208, 9008, 8304, 8224, 4112]
    # places of a share, 16 + tiles a head; 7 heads of 16 + 256, and 126 tiles: 2,045 before the first token, 2,048 are four to each of 512 workgroups
    rows = [8160, 8190, 8191, 8161, 8192, 8170, 8185, 4030]
    assert sum(16 + (n + 31) // 32 for n in rows) <= 2048 < sum(16 + (n + steps + 31) // 32 for n in rows)
    ctx = U.context(B, Hkv, G, max(caps))
    rope = hc.hc_rope_init(hc.HC_ROPE_HALF, 128, 10000.0)
    g = torch.Generator(device=U.DEV).manual_seed(7)
    a, b = (table_of(ctx, caps) for _ in range(2))
    a.state.copy_(torch.tensor([[n, n + 5] for n in rows], dtype=torch.int32))
    for i, n in enumerate(rows):
        for v in (0, 1):
            a.put(i, v, 0, torch.randn((n, D), generator=g, device=U.DEV).to(torch.bfloat16))
    a.acc.copy_(torch.rand((a.rows,), generator=g, device=U.DEV))
    for k in ("arena", "state", "acc"):
        getattr(b, k).copy_(getattr(a, k))
    small = [table_of(ctx, [512] * 8, [500, 100, 512, 30, 21, 400, 300, 20]) for _ in range(2)]
    for t in small[:1]:
        for k in ("arena", "state", "acc"):
            getattr(small[1], k).copy_(getattr(t, k))
    work = [a.work(), b.work()]
    x = torch.zeros((B, Hq + 2 * Hkv, D), dtype=torch.bfloat16, device=U.DEV)
    parts = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    q = [torch.zeros((B, Hq, D), dtype=torch.bfloat16, device=U.DEV) for _ in range(2)]
    out = [torch.zeros((B, Hq, D), device=U.DEV) for _ in range(2)]
    lse = [torch.zeros((B, Hq), device=U.DEV) for _ in range(2)]

    def step(c, i):
        hc.hc_kvq_append(ctx, c.kvq, rope, *parts, q[i], c.arena, c.state, c.acc)
        hc.hc_kvq_attn(ctx, c.kvq, c.arena, c.state, q[i], out[i], lse[i], c.acc, 0.9, work[i], work[i].numel())

    def evict(c, i):
        hc.hc_kvq_evict(ctx, c.kvq, c.arena, c.state, c.acc, small[i].kvq, small[i].arena, small[i].state, small[i].acc, None, work[i], work[i].numel())
    torch.cuda.synchronize()
    graph, gone = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(a, 0)
    with torch.cuda.graph(gone):
        evict(a, 0)
    torch.cuda.synchronize()
    for t in range(steps):
        x.copy_(torch.randn(x.shape, generator=g, device=U.DEV).to(torch.bfloat16))
        graph.replay()
        step(b, 1)
        assert torch.equal(out[0], out[1]) and torch.equal(lse[0], lse[1]) and torch.equal(q[0], q[1]), t
        assert torch.equal(a.state, b.state) and torch.equal(a.acc, b.acc), t
        if t % 11 == 3:
            gone.replay()                        # (beside the step's graph: the same work buffer)
            evict(b, 1)
            torch.cuda.synchronize()
            for k in ("arena", "state", "acc"):
                assert torch.equal(getattr(small[0], k), getattr(small[1], k)), (t, k)
    assert a.state[:, 0].tolist() == [min(n + steps, cap) for n, cap in zip(rows, caps)] and torch.equal(a.arena, b.arena)
    for i, n in enumerate(a.state[:, 0].tolist()):
        S.check_rms(out[0].view(8, G, D)[i], lse[0].view(8, G)[i], None, (0.0 + q[0].view(8, G, D)[i]), a.held(i, 0, n), a.held(i, 1, n), i)
    del graph, gone
    for c in (a, b, *small):
        c.close()
    hc.hc_destroy(ctx)


def test_captured_store_and_load():
    """A captured store appends the same prompt rows again with every replay, until a head has no more room; a captured load gives the same rows back, as they are then."""
    B, Hkv, count, caps = 2, 2, [70, 5], [192, 160, 16, 64]
    for count, caps in (([70, 5], [192, 160, 16, 64]), ([30, 7], [96, 80, 16, 32])):        # (several workgroups to a sequence, and a count behind them; one)
        ctx = U.context(B, Hkv, 2, 256)
        a, b = U.Cache(ctx, caps), U.Cache(ctx, caps)
        kv = torch.zeros((8 * 128 * D,), dtype=torch.bfloat16, device=U.DEV)
        k_off, v_off = [2 * i * 128 * D for i in range(4)], [(2 * i + 1) * 128 * D for i in range(4)]
        back = [torch.zeros((8 * 192 * D,), dtype=torch.bfloat16, device=U.DEV) for _ in range(2)]
        bk, bv = [2 * i * 192 * D for i in range(4)], [(2 * i + 1) * 192 * D for i in range(4)]

        def store(c):
            hc.hc_kvq_store(ctx, c.kvq, kv, k_off, v_off, [3, 0], count, c.arena, c.state, c.acc)  # noqa: B023

        def load(c, to):
            hc.hc_kvq_load(ctx, c.kvq, c.arena, c.state, [1, 0], [190, 40], to, bk, bv)  # noqa: B023
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            store(a)
            load(a, back[0])
        torch.cuda.synchronize()
        for t in range(4):
            kv.copy_(U.rows_of(8 * 128, 40 + t).view(-1))
            graph.replay()
            store(b)
            load(b, back[1])
            torch.cuda.synchronize()
            for k in ("arena", "state", "acc"):
                assert torch.equal(getattr(a, k), getattr(b, k)), (t, k)
            assert torch.equal(back[0], back[1]), t
            n = [min(caps[i], (t + 1) * count[i // 2]) for i in range(4)]
            assert a.state.tolist() == [[n[i], [3, 0][i // 2] + count[i // 2]] for i in range(4)]
            x = kv[k_off[0] + 3 * D:k_off[0] + (3 + count[0]) * D].view(-1, D)
            here = min(count[0], n[0] - t * count[0])
            if here > 0:
                assert torch.equal(a.held(0, 0, n[0])[t * count[0]:], U.decode(*U.encode(x[:here])))
        del graph
        a.close()
        b.close()
        hc.hc_destroy(ctx)
