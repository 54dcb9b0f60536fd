"""Rows into the cache held in 4 bits and back: a prompt's, the decode token's."""
import math

import pytest
import torch

import kvq_util as U
from paper_2601_13684_amd import binding as hc

pytestmark = pytest.mark.gpu
D = 128


def buffer_of(room, Hkv, gap=8):
    k_off, v_off, at = [], [], gap
    for n in room:
        for _ in range(Hkv):
            k_off.append(at)
            v_off.append(at + n * D + gap)
            at += 2 * (n * D + gap)
    return k_off, v_off, at


def outside(cache, written):
    """True where no head's first `written` rows are."""
    free = torch.ones((cache.bytes,), dtype=torch.bool, device=cache.arena.device)
    for i, (a, b) in enumerate(written):
        cap, off = cache.caps[i], cache.heads[i].off
        for at, size in ((0, 64), (64 * cap, 4), (68 * cap, 64), (132 * cap, 4)):
            free[off + at + size * a:off + at + size * b] = False
    return free


@pytest.mark.parametrize("kind", ["plain", "borders", "tiny", "huge", "odd"])
@pytest.mark.parametrize("Hkv,before,count,caps", [
    (2, [5], [1], [16]), (1, [0, 3, 0], [0, 13, 64], [64, 16, 64]), (2, [0, 7], [65, 200], [80, 208]), (8, [100], [129], [240]),
    (3, [10, 0, 2, 0], [30, 9, 0, 70], [32, 16, 16, 64])])
def test_store_and_load(kind, Hkv, before, count, caps):
    B = len(count)
    ctx = U.context(B, Hkv, 2, 512)
    cache = U.Cache(ctx, [c for c in caps for _ in range(Hkv)], rows=[n for n in before for _ in range(Hkv)], pos=[n + 1 for n in before for _ in range(Hkv)])
    room = [b + 1 + n for b, n in zip(before, count)]
    k_off, v_off, size = buffer_of(room, Hkv)
    kv = U.rows_of((size + D) // D, 3, kind).view(-1)[:size].clone()
    was, acc_was = cache.arena.clone(), cache.acc.clone()
    first = [b + 1 for b in before]                      # (not as many as there are rows: what an eviction leaves)
    hc.hc_kvq_store(ctx, cache.kvq, kv, k_off, v_off, first, count, cache.arena, cache.state, cache.acc)
    new = [(b, min(b + n, cap)) for b, n, cap in zip(before, count, caps) for _ in range(Hkv)]
    state = cache.state.tolist()
    for i, (a, b) in enumerate(new):
        s = i // Hkv
        assert state[i] == [b, first[s] + count[s]], i
        for v, off in ((0, k_off[i]), (1, v_off[i])):
            x = kv[off + first[s] * D:off + (first[s] + count[s]) * D].view(-1, D)[:b - a]
            codes, scales = cache.blocks(i, v)
            want = U.encode(x)
            assert torch.equal(scales[a:b], want[1]) and torch.equal(codes[a:b], want[0]), (i, v)
        r = cache.heads[i].row_off
        acc_was[r + a:r + b] = 0
    assert torch.equal(cache.acc, acc_was)
    free = outside(cache, new)
    assert torch.equal(cache.arena[free], was[free])
    # ---- and back: more rows asked for than there are
    out_k, out_v, size = buffer_of([n + 9 for n in caps], Hkv)
    back = torch.full((size,), 3.25, dtype=torch.bfloat16, device=U.DEV)
    f = [max(0, b - 2) for b in before]
    ask = [cap + 5 for cap in caps]
    hc.hc_kvq_load(ctx, cache.kvq, cache.arena, cache.state, f, ask, back, out_k, out_v)
    want = torch.full_like(back, 3.25)
    for i, (a, b) in enumerate(new):
        for v, off in ((0, out_k[i]), (1, out_v[i])):
            x = cache.held(i, v)[f[i // Hkv]:b]
            want[off:off + x.numel()] = x.to(torch.bfloat16).view(-1)
    known = torch.ones((size,), dtype=torch.bool, device=U.DEV)
    for i, (a, b) in enumerate(new):                    # (rows before the stored ones are the pattern's: not numbers that anyone put there)
        for off in (out_k[i], out_v[i]):
            known[off:off + max(0, before[i // Hkv] - f[i // Hkv]) * D] = False
    assert torch.equal(torch.nan_to_num(back[known], 1.5), torch.nan_to_num(want[known], 1.5)) and torch.equal(back[known].isnan(), want[known].isnan())
    cache.close()
    hc.hc_destroy(ctx)


@pytest.mark.parametrize("uneven", [False, True])
def test_many_sequences(uneven):
    """More than a launch takes, heads' blocks evenly apart or not."""
    B, Hkv = 150, 3
    count = [(7 * b) % 5 for b in range(B)]
    ctx = U.context(B, Hkv, 1, 64)
    cache = U.Cache(ctx, [16] * (B * Hkv), rows=[i % 3 for i in range(B * Hkv)])
    before = cache.state.clone()
    k_off, v_off, size = buffer_of([8] * B, Hkv)
    if uneven:                                           # the first and the last block of every sequence change places
        for off in (k_off, v_off):
            for b in range(B):
                off[b * Hkv], off[b * Hkv + 1] = off[b * Hkv + 1], off[b * Hkv]
    kv = U.rows_of((size + D) // D, 5).view(-1)[:size].clone()
    hc.hc_kvq_store(ctx, cache.kvq, kv, k_off, v_off, [1] * B, count, cache.arena, cache.state)
    back = torch.zeros_like(kv)
    hc.hc_kvq_load(ctx, cache.kvq, cache.arena, cache.state, [0] * B, [8] * B, back, k_off, v_off)
    for i in range(B * Hkv):
        n, c = int(before[i, 0]), count[i // Hkv]
        assert cache.state[i].tolist() == ([n + c, 1 + c] if c else before[i].tolist())
        for v, off in ((0, k_off[i]), (1, v_off[i])):
            x = kv[off + D:off + (1 + c) * D].view(c, D)
            want = U.encode(x)
            got = cache.blocks(i, v)
            assert torch.equal(got[0][n:n + c], want[0]) and torch.equal(got[1][n:n + c], want[1])
            assert torch.equal(back[off + n * D:off + (n + c) * D].double().view(c, D), U.decode(*want))
            assert (back[off + (n + c) * D:off + 8 * D] == 0).all()
    cache.close()
    hc.hc_destroy(ctx)


def test_every_bf16_value():
    """Every finite number as the largest of its group, and beside one that sets a scale far above its own."""
    x = torch.arange(65536, dtype=torch.int32, device=U.DEV).to(torch.int16).view(torch.bfloat16)
    x = x[torch.isfinite(x)]
    rows = torch.zeros((len(x), 4, 32), dtype=torch.bfloat16, device=U.DEV)
    rows[:, 0, 5], rows[:, 1, 31], rows[:, 1, 0], rows[:, 2], rows[:, 3, 7] = x, x, 6.0, x[:, None], x
    rows[:, 3, 8] = 2.0 ** -124
    rows = rows.view(-1, D)
    n = len(rows)
    ctx = U.context(1, 1, 1, n + 64)
    cap = (n + 15) // 16 * 16
    cache = U.Cache(ctx, [cap])
    kv = torch.cat([rows.view(-1), rows.flip(0).reshape(-1)])
    hc.hc_kvq_store(ctx, cache.kvq, kv, [0], [n * D], [0], [n], cache.arena, cache.state)
    for v, y in ((0, rows), (1, rows.flip(0))):
        want = U.encode(y)
        got = cache.blocks(0, v)
        assert torch.equal(got[1][:n], want[1]) and torch.equal(got[0][:n], want[0])
    cache.close()
    hc.hc_destroy(ctx)


@pytest.mark.parametrize("B,Hkv,G,rot,layout,norm,kind,gain", [
    (1, 2, 4, 128, hc.HC_ROPE_HALF, True, torch.bfloat16, 1.0), (3, 1, 8, 64, hc.HC_ROPE_INTERLEAVED, False, torch.float32, 1.0),
    (5, 2, 1, 32, hc.HC_ROPE_HALF, True, torch.float32, 0.75), (2, 8, 2, 96, hc.HC_ROPE_INTERLEAVED, True, torch.bfloat16, 1.25),
    (2, 3, 4, 0, hc.HC_ROPE_HALF, False, torch.bfloat16, 1.0), (1, 1, 1, 8, hc.HC_ROPE_HALF, True, torch.float32, 1.0)])
def test_append(B, Hkv, G, rot, layout, norm, kind, gain):
    """Keys and queries are the 64-bit ones rounded once to bf16 (a value next to the middle between two of bf16 is not in these inputs); rows the nearest of those."""
    ctx = U.context(B, Hkv, G, 256)
    Hq = Hkv * G
    before = [(7 * b) % 15 for b in range(B)]
    pos = [b * 40001 + 3 for b in range(B)]
    cache = U.Cache(ctx, [16] * (B * Hkv), rows=[n for n in before for _ in range(Hkv)], pos=[p for p in pos for _ in range(Hkv)])
    g = torch.Generator(device=U.DEV)
    g.manual_seed(B * 100 + rot)
    x = (torch.randn((B, Hq + 2 * Hkv + 1, D), generator=g, device=U.DEV) * 1.3).to(kind)
    w = [1 + 0.2 * torch.randn((D,), generator=g, device=U.DEV) for _ in range(2)] if norm else [None, None]
    rope = hc.hc_rope_init(layout, rot, 500000.0, q_norm=w[0], k_norm=w[1], eps=1e-5, gain=gain)
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:Hq + 2 * Hkv]
    q_out = torch.zeros((B, Hq, D), dtype=torch.bfloat16, device=U.DEV)
    was, acc_was = cache.arena.clone(), cache.acc.clone()
    hc.hc_kvq_append(ctx, cache.kvq, rope, q, k, v, q_out, cache.arena, cache.state, cache.acc)

    def turned(x, w):
        x = x.double()
        if w is not None:
            x = x * ((x * x).mean(-1, keepdim=True) + float(rope.eps)) ** -0.5 * w.double()
        y = x.clone()
        i = torch.arange(rot // 2, device=U.DEV)
        f = torch.tensor([rope.freq[j] for j in range(rot // 2)], dtype=torch.float64, device=U.DEV)
        a = torch.tensor(pos, dtype=torch.float64, device=U.DEV)[:, None, None] * f
        one, two = (i, i + rot // 2) if layout == hc.HC_ROPE_HALF else (2 * i, 2 * i + 1)
        y[..., one] = gain * (x[..., one] * a.cos() - x[..., two] * a.sin())
        y[..., two] = gain * (x[..., two] * a.cos() + x[..., one] * a.sin())
        return y

    def rounded(y):                                      # to bf16, once: 8 bits, ties to even
        m, e = torch.frexp(y)
        return torch.ldexp(torch.round(m * 256) / 256, e).to(torch.bfloat16)
    assert torch.equal(q_out, rounded(turned(q, w[0])))
    ks, vs = rounded(turned(k, w[1])), rounded(v.double())
    for b in range(B):
        for h in range(Hkv):
            i, n = b * Hkv + h, before[b]
            for side, y in ((0, ks), (1, vs)):
                codes, scales = cache.blocks(i, side)
                want = U.encode(y[b, h][None])
                assert torch.equal(scales[n], want[1][0]) and torch.equal(codes[n], want[0][0]), (b, h, side)
            acc_was[cache.heads[i].row_off + n] = 0
    assert cache.state.tolist() == [[before[i // Hkv] + 1, pos[i // Hkv] + 1] for i in range(B * Hkv)]
    assert torch.equal(cache.acc, acc_was)
    free = outside(cache, [(before[i // Hkv], before[i // Hkv] + 1) for i in range(B * Hkv)])
    assert torch.equal(cache.arena[free], was[free])
    cache.close()
    hc.hc_destroy(ctx)


def test_full_heads_and_states_out_of_range():
    """A head without room keeps its rows, its position moves on; counts beyond the room are taken as the room."""
    ctx = U.context(1, 4, 1, 64)
    cache = U.Cache(ctx, [16, 16, 32, 16], rows=[16, 15, 32, 400], pos=[90] * 4)
    x = U.rows_of(12, 1).view(1, 12, D)
    was = cache.arena.clone()
    q_out = torch.zeros((1, 4, D), dtype=torch.bfloat16, device=U.DEV)
    rope = hc.hc_rope_init(hc.HC_ROPE_HALF, 128, 10000.0)
    hc.hc_kvq_append(ctx, cache.kvq, rope, x[:, :4], x[:, 4:8], x[:, 8:], q_out, cache.arena, cache.state, cache.acc)
    assert cache.state.tolist() == [[16, 91], [16, 91], [32, 91], [16, 91]]
    free = outside(cache, [(0, 0), (15, 16), (0, 0), (0, 0)])
    assert torch.equal(cache.arena[free], was[free])
    assert (q_out != 0).any(-1).all()
    kv = U.rows_of(8 * 40, 2).view(-1)
    off = [i * 80 * D for i in range(4)]
    hc.hc_kvq_store(ctx, cache.kvq, kv, off, [o + 40 * D for o in off], [0], [40], cache.arena, cache.state, cache.acc)
    assert cache.state.tolist() == [[16, 40], [16, 40], [32, 40], [16, 40]]
    assert torch.equal(cache.arena[free], was[free])
    cache.close()
    hc.hc_destroy(ctx)
