"""A layer made from a prompt: its cache, host tier and lists, and what the decode tokens do to its compressed heads.  Run with `-m gpu` on an MI355X."""
import pytest
import torch

from paper_2601_13684_amd import binding as hc
from paper_2601_13684_amd import inputs as I
from paper_2601_13684_amd import runtime as R

import prompt_util as P

pytestmark = pytest.mark.gpu
DEV, D = P.DEV, P.D
SINK, RECENT, BUDGET = 8, 32, 200


def make(G, steps, dtype, layout, seed=21):
    """A prompt that has taken its tokens in three chunks, the last tokens' queries, and the rows of the tokens that follow."""
    Hkv, lens = 2, [700, 1023]
    heads = [[I.HeadSpec(I.ROLE_FULL), I.HeadSpec(I.ROLE_SATELLITE, rep=0, sink=SINK, recent=RECENT, budget=BUDGET)]] * 2
    spec = I.LayerSpec(B=2, Hq=Hkv * G, Hkv=Hkv, D=D, ctx=lens, heads=heads)
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    x = [torch.randn((n + steps, Hkv * (G + 2), D), generator=g, device=DEV).to(dtype) for n in lens]
    rope = hc.hc_rope_init(layout, 128, 10000.0, k_norm=1 + 0.1 * torch.randn((D,), generator=g, device=DEV))
    split = lambda rows: (rows[:, :Hkv * G], rows[:, Hkv * G:-Hkv], rows[:, -Hkv:])  # noqa: E731
    ctx = R.Context(R.make_config(spec, growth=steps), DEV)
    prompt, got = R.Prompt(ctx, lens), [[], []]
    for count in ([300, 1], [0, 1000], [400, 22]):
        chunk = prompt.chunk(rope, *split(torch.cat([x[b][prompt.length[b]:prompt.length[b] + count[b]] for b in range(2)])), count)
        for b in range(2):
            got[b].append([t.split(count)[b] for t in chunk])
    q, out, lse = ([torch.cat([c[i] for c in got[b]]) for b in range(2)] for i in range(3))
    later = [split(torch.stack([x[b][lens[b] + t] for b in range(2)])) for t in range(steps)]
    return spec, ctx, prompt, rope, q, out, lse, later


def rows_of(prompt, spec, b, h):
    n, i = spec.ctx[b], b * spec.Hkv + h
    return [prompt.kv[o[i]:o[i] + n * D].view(n, D) for o in (prompt.k_off, prompt.v_off)]


def block(lay, b, h, rows):
    d = lay.descs[b * lay.spec.Hkv + h]
    return [lay.arena[o:o + rows * D].view(rows, D) for o in (d.k_off, d.v_off)]


@pytest.mark.parametrize("G", [1, 4])
def test_outputs_and_lse_of_chunks(G):
    """Of every chunk, behind what the chunks before it left."""
    spec, ctx, prompt, rope, q, out, lse, _ = make(G, 0, torch.bfloat16, hc.HC_ROPE_HALF)
    torch.cuda.synchronize()
    for b, n in enumerate(spec.ctx):
        at = slice(b * spec.Hkv, (b + 1) * spec.Hkv)
        P.check_attention(out[b], lse[b], P.attention(q[b], prompt.kv, prompt.k_off[at], prompt.v_off[at], [0], [n], spec.Hkv, G), b)
    ctx.close()


@pytest.mark.parametrize("G,dtype,layout", [(4, torch.bfloat16, hc.HC_ROPE_HALF), (8, torch.float32, hc.HC_ROPE_INTERLEAVED)])
def test_a_layer_made_from_a_prompt(G, dtype, layout):
    """The same, to the bit, as one made from the prompt's rows as data; its compressed heads hold the rows that their lists name."""
    spec, ctx, prompt, rope, q, _, _, _ = make(G, 3, dtype, layout)
    last = torch.stack([q[b][-1] for b in range(2)])
    data = I.LayerData()
    for b in range(2):
        for h in range(2):
            data.K[(b, h)], data.V[(b, h)] = (r.clone() for r in rows_of(prompt, spec, b, h))
    one, two = (R.LayerRuntime(ctx, spec, d, None, None, growth=3, prefill=(last, 1)) for d in (prompt, data))
    torch.cuda.synchronize()
    for name in ("arena", "tier", "topk_idx", "base_idx", "slot_pos", "ring"):
        assert torch.equal(getattr(one, name), getattr(two, name)), name
    r = BUDGET - SINK - RECENT
    for b, n in enumerate(spec.ctx):
        for mine, row in zip(block(one, b, 0, n), rows_of(prompt, spec, b, 0)):
            assert torch.equal(mine, row)
        held = one.slot_pos[2 * b + 1, :r].long()
        assert (held[1:] > held[:-1]).all() and held[0] >= SINK and held[-1] < n - RECENT
        at = torch.cat([torch.arange(SINK, device=DEV), torch.arange(n - RECENT, n, device=DEV), held])
        for mine, row in zip(block(one, b, 1, BUDGET), rows_of(prompt, spec, b, 1)):
            assert torch.equal(mine, row[at])
        d = one.descs[2 * b + 1]
        assert torch.equal(one.tier[d.tier_off:d.tier_off + n * 2 * D].view(n, 2, D), torch.stack(rows_of(prompt, spec, b, 1), 1).cpu())
    with pytest.raises(ValueError):
        one.prefill_from(R.Prompt(ctx, spec.ctx), last)              # one that has taken nothing
    for c in (one, two, ctx):
        c.close()


@pytest.mark.parametrize("G,dtype,layout", [(4, torch.bfloat16, hc.HC_ROPE_HALF), (8, torch.float32, hc.HC_ROPE_INTERLEAVED)])
def test_tokens_in_a_compressed_head(G, dtype, layout):
    """More of them than the recent window holds: every token's rows in the arena and in the host tier, and attention over exactly the resident rows."""
    steps = RECENT + 5
    spec, ctx, prompt, rope, q, _, _, later = make(G, steps, dtype, layout)
    lay = R.LayerRuntime(ctx, spec, prompt, None, None, growth=steps, prefill=(torch.stack([q[b][-1] for b in range(2)]), 1))
    torch.cuda.synchronize()
    # the rows that the head has, slot by slot, followed from token to token
    slots = [[r.clone() for r in block(lay, b, 1, BUDGET)] for b in range(2)]
    tier = [torch.stack(rows_of(prompt, spec, b, 1), 1) for b in range(2)]
    w = rope.keep[1]
    for t in range(steps):
        qt = lay.append_rope(rope, *later[t])
        lay.attn(qt)
        torch.cuda.synchronize()
        for b, n in enumerate(spec.ctx):
            pos = torch.full((1,), n + t, device=DEV)
            K, V = block(lay, b, 1, BUDGET)
            slot = SINK + t % RECENT
            P.check_turned(K[slot][None], *(y[:, 0] for y in P.turned(later[t][1][b:b + 1, 1:], w, rope.eps, pos, rope)), ("k", t, b))
            assert torch.equal(V[slot], later[t][2][b, 1].to(torch.bfloat16))
            slots[b][0][slot], slots[b][1][slot] = K[slot], V[slot]
            assert torch.equal(K, slots[b][0]) and torch.equal(V, slots[b][1])          # no other slot
            tier[b] = torch.cat([tier[b], torch.stack([K[slot], V[slot]])[None]])
            s = qt[b, G:].double() @ K.double().t() / D ** 0.5
            o = torch.softmax(s, -1) @ V.double()
            assert ((lay.out[b, G:].double() - o).abs() <= 1e-5 + 1e-5 * V.double().abs().max()).all()
            l = torch.logsumexp(s, -1)
            assert ((lay.lse[b, G:].double() - l).abs() <= 1e-4 + 1e-6 * l.abs()).all()
    for b, n in enumerate(spec.ctx):
        d = lay.descs[2 * b + 1]
        assert torch.equal(lay.tier[d.tier_off:d.tier_off + (n + steps) * 2 * D].view(-1, 2, D), tier[b].cpu())
    lay.close()
    ctx.close()
