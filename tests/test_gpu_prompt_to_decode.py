"""A layer from its projections on: a prompt in chunks (rotation, attention), the cache built from it, tokens appended with rotation and attended over.
Run with `-m gpu` on an MI355X."""
import pytest
import torch

from paper_2601_13684_amd import binding as hc
from paper_2601_13684_amd import inputs as I
from paper_2601_13684_amd import runtime as R

import prompt_util as P

pytestmark = pytest.mark.gpu
DEV, D = P.DEV, P.D


@pytest.mark.parametrize("G,layout,dtype", [(4, hc.HC_ROPE_HALF, torch.bfloat16), (8, hc.HC_ROPE_INTERLEAVED, torch.float32)])
def test_chunks_cache_and_tokens(G, layout, dtype):
    print("prompt to decode", G, layout, dtype, flush=True)
    Hkv, ctx_lens, steps = 2, [700, 1023], 5
    heads = [[I.HeadSpec(I.ROLE_FULL), I.HeadSpec(I.ROLE_SATELLITE, rep=0, sink=8, recent=32, budget=200)]] * 2
    spec = I.LayerSpec(B=2, Hq=Hkv * G, Hkv=Hkv, D=D, ctx=ctx_lens, heads=heads)
    Hq = spec.Hq
    g = torch.Generator(device=DEV)
    g.manual_seed(11)
    total = [n + steps for n in ctx_lens]
    x = [torch.randn((n, Hq + 2 * Hkv, D), generator=g, device=DEV).to(dtype) for n in total]
    w = [1 + 0.1 * torch.randn((D,), generator=g, device=DEV) for _ in range(2)]
    rope = hc.hc_rope_init(layout, 128, 10000.0, q_norm=w[0], k_norm=w[1])
    ctx = R.Context(R.make_config(spec, growth=steps), DEV)
    prompt = R.Prompt(ctx, ctx_lens)
    # the plain form: 64 bits, rows rounded to bf16 where the path rounds them
    plain = []
    for b, n in enumerate(total):
        pos = torch.arange(n, device=DEV)
        q, k = (P.turned(x[b][:, s], wt, rope.eps, pos, rope)[0].to(torch.bfloat16) for s, wt in ((slice(0, Hq), w[0]), (slice(Hq, Hq + Hkv), w[1])))
        plain.append((q, k, x[b][:, Hq + Hkv:].to(torch.bfloat16)))
    outs, qs = [[], []], [[], []]
    for count in ([1, 500], [400, 0], [299, 523]):
        rows = torch.cat([x[b][prompt.length[b]:prompt.length[b] + count[b]] for b in range(2)])
        q, out, lse = prompt.chunk(rope, rows[:, :Hq], rows[:, Hq:Hq + Hkv], rows[:, Hq + Hkv:], count)
        for b, (qq, oo) in enumerate(zip(q.split(count), out.split(count))):
            qs[b].append(qq)
            outs[b].append(oo)
    torch.cuda.synchronize()
    assert prompt.length == ctx_lens
    for b, n in enumerate(ctx_lens):
        q = torch.cat(qs[b])
        # what was rotated differs from the plain rows by a rounding that fell the other way at most; attention is held to what it was given
        assert ((q.double() - plain[b][0][:n].double()).abs() <= 2.0 ** -7 * plain[b][0][:n].double().abs() + 1e-4).all()
        offs = prompt.k_off[b * Hkv:(b + 1) * Hkv], prompt.v_off[b * Hkv:(b + 1) * Hkv]
        want = P.attention(q, prompt.kv, *offs, [0], [n], Hkv, G)
        P.check_attention(torch.cat(outs[b]), want[1].float(), want, b)
    lay = layer_from(ctx, spec, prompt, torch.stack([qs[b][-1][-1] for b in range(2)]), steps)
    for t in range(steps):
        rows = torch.stack([x[b][ctx_lens[b] + t] for b in range(2)])
        q = lay.append_rope(rope, rows[:, :Hq], rows[:, Hq:Hq + Hkv], rows[:, Hq + Hkv:])
        lay.attn(q)
        torch.cuda.synchronize()
        for b in range(2):
            n = ctx_lens[b] + t + 1
            d = lay.descs[b * Hkv]
            K, V = (lay.arena[o:o + n * D].view(n, D) for o in (d.k_off, d.v_off))
            assert ((K.double() - plain[b][1][:n, 0].double()).abs() <= 2.0 ** -7 * plain[b][1][:n, 0].double().abs() + 1e-4).all()
            assert torch.equal(V, plain[b][2][:n, 0])
            s = q[b, :G].double() @ K.double().t() / D ** 0.5
            o = torch.softmax(s, -1) @ V.double()
            assert ((lay.out[b, :G].double() - o).abs() <= 1e-5 + 1e-5 * V.double().abs().max()).all()
    lay.close()
    ctx.close()


def layer_from(ctx, spec, prompt, q_last, growth):
    """A layer whose state hc_prefill_init builds from what the prompt left."""
    n = [torch.zeros((c, D), dtype=torch.bfloat16) for c in spec.ctx]
    data = I.LayerData({(b, h): n[b] for b in range(spec.B) for h in range(spec.Hkv)}, {(b, h): n[b] for b in range(spec.B) for h in range(spec.Hkv)}, {})
    lay = R.LayerRuntime(ctx, spec, data, None, None, growth=growth, prefill=(q_last, 1))
    lay.prefill_from(prompt, q_last)
    return lay


def test_chunks_on_another_stream():
    """Everything that a chunk allocates and launches is the given stream's: as on the current one, with the current one's work around it."""
    Hkv, G, ctx_lens = 2, 4, [300, 1100]
    spec = I.LayerSpec(B=2, Hq=Hkv * G, Hkv=Hkv, D=D, ctx=ctx_lens, heads=[[I.HeadSpec(I.ROLE_FULL)] * 2] * 2)
    ctx = R.Context(R.make_config(spec), DEV)
    rope = hc.hc_rope_init(hc.HC_ROPE_HALF, 64, 10000.0)
    x = torch.randn((sum(ctx_lens), Hkv * (G + 2), D), device=DEV).to(torch.bfloat16)
    qkv = x[:, :Hkv * G], x[:, Hkv * G:-Hkv], x[:, -Hkv:]
    want = R.Prompt(ctx, ctx_lens).chunk(rope, *qkv, ctx_lens)
    for make in (lambda s: s, lambda s: s.cuda_stream):
        prompt, side = R.Prompt(ctx, ctx_lens), torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        got = prompt.chunk(rope, *qkv, ctx_lens, stream=make(side))
        noise = [torch.full_like(t, 3.0) for t in want]          # the current stream's next allocations are not the chunk's memory
        side.synchronize()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)) and all((n == 3).all() for n in noise)
