"""hc_prefill_rope and hc_append_rope against the 64-bit form.  Run with `-m gpu` on an MI355X."""
import pytest
import torch

from paper_2601_13684_amd import binding as hc
from paper_2601_13684_amd import inputs as I
from paper_2601_13684_amd import runtime as R

import prompt_util as P

pytestmark = pytest.mark.gpu
DEV, D = P.DEV, P.D
BANDS = dict(kind=hc.HC_ROPE_BANDS, original=8192, factor=8.0, low=1.0, high=4.0)


def rope_of(layout, rot, theta=10000.0, scaling=None, norm=True, gain=None, seed=3):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    w = [1 + 0.3 * torch.randn((D,), generator=g, device=DEV) for _ in range(2)] if norm else [None, None]
    return hc.hc_rope_init(layout, rot, theta, hc.hc_rope_scaling(**scaling) if scaling else None, q_norm=w[0], k_norm=w[1], eps=1e-5, gain=gain), w


def projected(T, Hq, Hkv, dtype, seed, fused=True):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    x = (torch.randn((T, Hq + 2 * Hkv, D), generator=g, device=DEV) * torch.exp(torch.randn((Hq + 2 * Hkv, D), generator=g, device=DEV))).to(dtype)
    if fused:
        return x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    return x[:, :Hq].contiguous(), x[:, Hq:Hq + Hkv].contiguous(), x[:, Hq + Hkv:].contiguous()


def check_prefill(first, count, Hkv, G, rope, w, dtype, fused=True, gap=8, room=2):
    print("rope", first, count, Hkv, G, rope.layout, rope.rot_dim, dtype, flush=True)
    T, B = sum(count), len(first)
    q, k, v = projected(T, Hkv * G, Hkv, dtype, T + Hkv, fused)
    k_off, v_off, size = P.blocks([f + n + room for f, n in zip(first, count)], Hkv, gap)
    kv = torch.full((size + 8,), 7.0, dtype=torch.bfloat16, device=DEV)
    q_out = torch.full((T + 1, Hkv * G, D), 7.0, dtype=torch.bfloat16, device=DEV)
    ctx = P.context(B, Hkv, G, max(f + n for f, n in zip(first, count)))
    hc.hc_prefill_rope(ctx, rope, q, k, v, first, count, q_out, kv, k_off, v_off)
    torch.cuda.synchronize()
    hc.hc_destroy(ctx)
    pos = torch.cat([torch.arange(f, f + n, device=DEV) for f, n in zip(first, count)])
    P.check_turned(q_out[:T], *P.turned(q, w[0], rope.eps, pos, rope), "q")
    assert (q_out[T:] == 7).all()
    ky, ks = P.turned(k, w[1], rope.eps, pos, rope)
    t = 0
    for b, (f, n) in enumerate(zip(first, count)):
        for h in range(Hkv):
            at, av = k_off[b * Hkv + h] + f * D, v_off[b * Hkv + h] + f * D
            P.check_turned(kv[at:at + n * D].view(n, D), ky[t:t + n, h], ks[t:t + n, h], ("k", b, h))
            assert torch.equal(kv[av:av + n * D].view(n, D), v[t:t + n, h].to(torch.bfloat16)), ("v", b, h)
            kv[at:at + n * D] = 7
            kv[av:av + n * D] = 7
        t += n
    assert (kv == 7).all()


@pytest.mark.parametrize("layout", [hc.HC_ROPE_HALF, hc.HC_ROPE_INTERLEAVED])
@pytest.mark.parametrize("rot", [0, 8, 24, 32, 64, 96, 120, 128])
@pytest.mark.parametrize("dtype,norm", [(torch.bfloat16, True), (torch.float32, False)])
def test_layouts_and_parts(layout, rot, dtype, norm):
    rope, w = rope_of(layout, rot, norm=norm, gain=1.25 if rot == 64 else None)
    check_prefill([0, 5000], [37, 3], 2, 4, rope, w, dtype)


@pytest.mark.parametrize("first,count,Hkv,G", [
    ([0], [1], 1, 1), ([7], [5], 1, 8), ([0, 3, 9], [0, 1, 0], 2, 2), ([131000], [72], 8, 4),
    ([11 * i for i in range(70)], [1 + i % 4 for i in range(70)], 2, 4), ([9 * i for i in range(33)], [(i * 7) % 20 for i in range(33)], 8, 1),
    ([3, 0], [40, 2], 128, 1), ([0], [2049], 8, 4)])
@pytest.mark.parametrize("fused", [True, False])
def test_packed(first, count, Hkv, G, fused):
    rope, w = rope_of(hc.HC_ROPE_HALF, 128, 500000.0, BANDS, norm=len(first) % 2 == 1)
    check_prefill(first, count, Hkv, G, rope, w, torch.bfloat16, fused)


@pytest.mark.parametrize("layout", [hc.HC_ROPE_HALF, hc.HC_ROPE_INTERLEAVED])
def test_far_positions(layout):
    """Positions up to 2^24 - 1: an angle in 32 bits would be off by half a radian."""
    rope, w = rope_of(layout, 128, norm=False)
    check_prefill([2 ** 24 - 5, 2 ** 23 + 1], [5, 3], 1, 1, rope, w, torch.float32, gap=0, room=0)


def test_one_row_for_all_tokens_and_one_norm():
    """A stride of 0 (the same heads at every position), and a norm for the queries alone."""
    rope, w = rope_of(hc.HC_ROPE_INTERLEAVED, 64)
    rope.k_norm = None
    T = 9
    q, k, v = (x.expand(T, -1, -1) for x in projected(1, 8, 2, torch.bfloat16, 4))
    k_off, v_off, size = P.blocks([T], 2)
    kv = torch.zeros((size,), dtype=torch.bfloat16, device=DEV)
    q_out = torch.zeros((T, 8, D), dtype=torch.bfloat16, device=DEV)
    ctx = P.context(1, 2, 4, T)
    hc.hc_prefill_rope(ctx, rope, q, k, v, [0], [T], q_out, kv, k_off, v_off)
    torch.cuda.synchronize()
    pos = torch.arange(T, device=DEV)
    P.check_turned(q_out, *P.turned(q, w[0], rope.eps, pos, rope), "q")
    ky, ks = P.turned(k, None, rope.eps, pos, rope)
    for h in range(2):
        P.check_turned(kv[k_off[h]:k_off[h] + T * D].view(T, D), ky[:, h], ks[:, h], "k")
        assert torch.equal(kv[v_off[h]:v_off[h] + T * D].view(T, D), v[:, h])
    hc.hc_destroy(ctx)


def test_rows_of_zeros_and_what_is_not_finite():
    """A row of zeros keeps to zeros under the norm; an infinity or a NaN stays inside its head."""
    rope, w = rope_of(hc.HC_ROPE_HALF, 128)
    q, k, v = projected(4, 4, 1, torch.bfloat16, 9, fused=False)
    q[0, 0] = 0
    q[1, 1, 3] = float("inf")
    q[2, 2, 100] = float("nan")
    k_off, v_off, size = P.blocks([4], 1)
    kv = torch.zeros((size,), dtype=torch.bfloat16, device=DEV)
    q_out = torch.zeros((4, 4, D), dtype=torch.bfloat16, device=DEV)
    ctx = P.context(1, 1, 4, 64)
    hc.hc_prefill_rope(ctx, rope, q, k, v, [0], [4], q_out, kv, k_off, v_off)
    torch.cuda.synchronize()
    bad = ~torch.isfinite(q_out.float()).all(-1)
    assert (q_out[0, 0] == 0).all() and bad[1, 1] and bad[2, 2] and int(bad.sum()) == 2
    hc.hc_destroy(ctx)


def test_graph_and_stream():
    rope, w = rope_of(hc.HC_ROPE_HALF, 128)
    q, k, v = projected(20, 8, 2, torch.bfloat16, 5, fused=False)
    k_off, v_off, size = P.blocks([30], 2)
    kv = torch.zeros((size,), dtype=torch.bfloat16, device=DEV)
    q_out = torch.zeros((20, 8, D), dtype=torch.bfloat16, device=DEV)
    ctx = P.context(1, 2, 4, 64)
    call = lambda s=None: hc.hc_prefill_rope(ctx, rope, q, k, v, [10], [20], q_out, kv, k_off, v_off, s)  # noqa: E731
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    call(s)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(3):
        q.copy_(torch.randn_like(q.float()).to(torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        got = q_out.clone(), kv.clone()
        q_out.zero_()
        kv.zero_()
        call()
        torch.cuda.synchronize()
        assert torch.equal(got[0], q_out) and torch.equal(got[1], kv)
    hc.hc_destroy(ctx)


# ---- the decode token ----------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("G", [1, 2, 4, 8])
@pytest.mark.parametrize("layout,rot,dtype,norm", [(hc.HC_ROPE_HALF, 128, torch.bfloat16, True), (hc.HC_ROPE_INTERLEAVED, 64, torch.float32, True),
                                                   (hc.HC_ROPE_HALF, 24, torch.float32, False)])
def test_append_is_rotation_and_append(G, layout, rot, dtype, norm):
    """The fused call leaves, to the bit, what hc_prefill_rope of the token and hc_append_kv of its rows leave: arena, host tier, lengths; for
    more tokens than the recent windows hold and than a plan lasts."""
    print("append", G, layout, rot, dtype, norm, flush=True)
    Hkv, B = 5, 2
    heads = [[I.HeadSpec(I.ROLE_FULL), I.HeadSpec(I.ROLE_SATELLITE, rep=0, sink=4, recent=9, budget=40), I.HeadSpec(I.ROLE_ANCHOR, sink=2, recent=0, budget=30),
              I.HeadSpec(I.ROLE_ANCHOR, sink=0, recent=70, budget=80), I.HeadSpec(I.ROLE_FULL)]] * B
    spec = I.LayerSpec(B=B, Hq=Hkv * G, Hkv=Hkv, D=D, ctx=[300, 411], heads=heads)
    data = I.LayerData()
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    for b in range(B):
        for h in range(Hkv):
            data.K[(b, h)] = torch.randn((spec.ctx[b], D), generator=g, device=DEV).to(torch.bfloat16)
            data.V[(b, h)] = torch.randn((spec.ctx[b], D), generator=g, device=DEV).to(torch.bfloat16)
    steps = 75
    rope, w = rope_of(layout, rot, norm=norm, scaling=dict(kind=hc.HC_ROPE_LINEAR, factor=2.0))
    ctx = R.Context(R.make_config(spec, growth=steps), DEV)
    q_last = torch.randn((B, spec.Hq, D), generator=g, device=DEV).to(torch.bfloat16)
    one, two = (R.LayerRuntime(ctx, spec, data, None, None, growth=steps, prefill=(q_last, 1)) for _ in range(2))
    k_off, v_off, size = P.blocks([spec.ctx[b] + steps for b in range(B)], Hkv)
    kv = torch.zeros((size,), dtype=torch.bfloat16, device=DEV)
    q2 = torch.zeros((B, spec.Hq, D), dtype=torch.bfloat16, device=DEV)
    for t in range(steps):
        q, k, v = projected(B, spec.Hq, Hkv, dtype, 100 + t, fused=t % 2 == 0)
        q1 = one.append_rope(rope, q, k, v)
        at = [spec.ctx[b] + t for b in range(B)]
        hc.hc_prefill_rope(ctx.handle, rope, q, k, v, at, [1] * B, q2, kv, k_off, v_off)
        rows = [torch.stack([kv[o[i] + at[i // Hkv] * D:][:D] for i in range(B * Hkv)]).view(B, Hkv, D) for o in (k_off, v_off)]
        two.append(*rows)
        assert torch.equal(q1, q2), t
        one.attn(q1)
        two.attn(q2)
    torch.cuda.synchronize()
    assert torch.equal(one.arena, two.arena) and torch.equal(one.tier, two.tier)
    assert torch.equal(one.out, two.out) and torch.equal(one.lse, two.lse)
    assert [one.context(b) for b in range(B)] == [spec.ctx[b] + steps for b in range(B)]
    q, k, v = projected(B, spec.Hq, Hkv, dtype, 7)
    with pytest.raises(hc.HcError) as e:                 # no room left
        one.append_rope(rope, q, k, v)
    assert e.value.status == hc.HC_ESHAPE and "hc_append_rope" in str(e.value)
    for x in (one, two, ctx):
        x.close()
