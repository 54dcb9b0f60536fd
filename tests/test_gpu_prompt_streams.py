"""The prompt stage on another stream than the one its buffers were made on.  Run with `-m gpu` on an MI355X."""
import pytest
import torch

from paper_2601_13684_amd import binding as hc
from paper_2601_13684_amd import inputs as I
from paper_2601_13684_amd import runtime as R

import prompt_util as P

pytestmark = pytest.mark.gpu
DEV, D = P.DEV, P.D


@pytest.mark.parametrize("bare", [False, True])
def test_made_and_dropped_while_the_other_stream_works(bare):
    """The current stream is busy when the buffers are made, the side stream does not wait for it by itself, and the Prompt is gone, its memory asked for
    and overwritten, before either is through."""
    Hkv, G, lens = 2, 4, [300, 5100]
    spec = I.LayerSpec(B=2, Hq=Hkv * G, Hkv=Hkv, D=D, ctx=lens, heads=[[I.HeadSpec(I.ROLE_FULL)] * 2] * 2)
    ctx = R.Context(R.make_config(spec), DEV)
    rope = hc.hc_rope_init(hc.HC_ROPE_HALF, 64, 10000.0)
    x = torch.randn((sum(lens), Hkv * (G + 2), D), device=DEV).to(torch.bfloat16)
    qkv = x[:, :Hkv * G], x[:, Hkv * G:-Hkv], x[:, -Hkv:]
    p = R.Prompt(ctx, lens)
    want = [t.clone() for t in (*p.chunk(rope, *qkv, lens), p.kv)]
    n_work, n_kv = p.work.numel(), p.kv.numel()
    del p
    side, busy = torch.cuda.Stream(), torch.empty((1 << 28,), dtype=torch.float32, device=DEV)
    for _ in range(3):
        torch.cuda.synchronize()
        for _ in range(40):
            busy.fill_(1.0)                      # milliseconds of work in front of the buffers' fill
        prompt = R.Prompt(ctx, lens)
        got = prompt.chunk(rope, *qkv, lens, stream=side.cuda_stream if bare else side)
        with torch.cuda.stream(side):
            kv = prompt.kv.clone()
        del prompt
        noise = [torch.full((n_work,), 255, dtype=torch.uint8, device=DEV), torch.full((n_kv,), 9.0, dtype=torch.bfloat16, device=DEV)]
        side.synchronize()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((*got, kv), want))
        del noise
    ctx.close()


def test_a_chunk_captured():
    """A capture runs on a stream of its own: replays beside eager chunks of another Prompt give the eager results."""
    Hkv, G, lens = 2, 4, [700]
    spec = I.LayerSpec(B=1, Hq=Hkv * G, Hkv=Hkv, D=D, ctx=lens, heads=[[I.HeadSpec(I.ROLE_FULL)] * 2])
    ctx = R.Context(R.make_config(spec), DEV)
    rope = hc.hc_rope_init(hc.HC_ROPE_INTERLEAVED, 128, 10000.0)
    x = torch.randn((700, Hkv * (G + 2), D), device=DEV).to(torch.bfloat16)
    qkv = x[:, :Hkv * G], x[:, Hkv * G:-Hkv], x[:, -Hkv:]
    prompt, graph = R.Prompt(ctx, lens), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = prompt.chunk(rope, *qkv, lens)
    for _ in range(3):
        x.copy_(torch.randn_like(x.float()).to(torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        eager = R.Prompt(ctx, lens).chunk(rope, *qkv, lens)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, eager))
    ctx.close()


@pytest.mark.parametrize("where", [0, "current"])
def test_a_chunk_on_the_default_stream(where):
    """By its handle, or as the current one of another stream's context."""
    lens = [200]
    spec = I.LayerSpec(B=1, Hq=4, Hkv=1, D=D, ctx=lens, heads=[[I.HeadSpec(I.ROLE_FULL)]])
    ctx = R.Context(R.make_config(spec), DEV)
    rope = hc.hc_rope_init(hc.HC_ROPE_HALF, 128, 10000.0)
    x = torch.randn((200, 6, D), device=DEV).to(torch.bfloat16)
    qkv = x[:, :4], x[:, 4:5], x[:, 5:]
    want = R.Prompt(ctx, lens).chunk(rope, *qkv, lens)
    torch.cuda.synchronize()
    if where == 0:
        got = R.Prompt(ctx, lens).chunk(rope, *qkv, lens, stream=0)
    else:
        prompt = R.Prompt(ctx, lens)
        with torch.cuda.stream(torch.cuda.Stream()):
            got = prompt.chunk(rope, *qkv, lens)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    ctx.close()


def test_a_layer_made_on_another_stream():
    """prefill_from on a side stream, the current one busy in front of the layer's own fills: the layer is what it is on the current stream."""
    Hkv, G, lens = 2, 4, [900]
    heads = [[I.HeadSpec(I.ROLE_FULL), I.HeadSpec(I.ROLE_SATELLITE, rep=0, sink=4, recent=16, budget=120)]]
    spec = I.LayerSpec(B=1, Hq=Hkv * G, Hkv=Hkv, D=D, ctx=lens, heads=heads)
    ctx = R.Context(R.make_config(spec), DEV)
    rope = hc.hc_rope_init(hc.HC_ROPE_HALF, 128, 10000.0)
    x = torch.randn((900, Hkv * (G + 2), D), device=DEV).to(torch.bfloat16)
    prompt = R.Prompt(ctx, lens)
    q, _, _ = prompt.chunk(rope, x[:, :Hkv * G], x[:, Hkv * G:-Hkv], x[:, -Hkv:], lens)
    want = R.LayerRuntime(ctx, spec, prompt, None, None, prefill=(q[-1:], 1))
    busy, side = torch.empty((1 << 28,), device=DEV), torch.cuda.Stream()
    zeros = {(0, h): torch.zeros((900, D), dtype=torch.bfloat16) for h in range(2)}
    for _ in range(3):
        torch.cuda.synchronize()
        for _ in range(40):
            busy.fill_(1.0)
        lay = R.LayerRuntime(ctx, spec, I.LayerData(zeros, zeros, {}), {(0, 1): torch.arange(4, 104)}, {})
        lay.prefill_from(prompt, q[-1:].cpu(), 1, side)
        side.synchronize()
        torch.cuda.synchronize()
        for name in ("arena", "tier", "topk_idx", "base_idx", "slot_pos", "ring"):
            assert torch.equal(getattr(lay, name), getattr(want, name)), name
        lay.close()
    want.close()
    ctx.close()
