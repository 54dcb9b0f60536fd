"""The operators in front of the decode path, as measurable cases: what happens to a prompt's tokens, and to the decode token, between the
projections and the cache.

Kinds of case:
  rope    hc_prefill_rope: norms and position rotation of a prompt's (or a chunk's) queries and keys; K and V rows to the prompt's buffer
  attn    hc_prefill_attn: causal attention of these queries over that buffer, packed sequences, grouped heads
  append  hc_append_rope: norms and rotation of the decode token, its K and V rows into the heterogeneous cache

``first`` tokens of a sequence are there before the call, ``count`` come with it (both: one number a sequence).  ``rot``: elements of a head that
rotate; ``pairs``: "half" (i, i + rot/2) or "interleaved" (2i, 2i + 1); ``scaling``: how the frequencies are fitted to long contexts.
"""
import math

import torch

own = False
DEV = "cuda:0"
D = 128
EPS = 1e-6
GROW = 98304         # tokens a measured cache has room for
SCALING = dict(linear=dict(factor=4.0), base=dict(factor=4.0), bands=dict(factor=8.0, low=1.0, high=4.0, original=8192))


def _case(name, kind, first, count, Hkv=8, G=4, **more):
    c = dict(kind=kind, first=first, count=count, Hkv=Hkv, G=G)
    if name:
        c["name"] = name
    c.update(more)
    return c


def listed():
    return [
        # A short chunk of one conversation, small layer: launch latency.
        _case("rope_17", "rope", "4001", "17", Hkv=2, rot=128, pairs="half", scaling="none", norm=True, type="bf16", theta=10000.0),
        # The prompt of the 32K configuration, one layer, frequencies in bands for a long context, no norms.
        _case("rope_32k", "rope", "0", "32003", rot=128, pairs="half", scaling="bands", norm=False, type="bf16", theta=500000.0),
        # A serving batch's ragged chunks behind contexts of different lengths; 32-bit projections, half of the head rotates.
        _case("rope_batch", "rope", "8192,0,30011,0,65536,12000,0,500", "1024,777,2048,33,1500,1,4096,2049", rot=64, pairs="interleaved", scaling="linear",
              norm=True, type="f32", theta=10000.0),
        # One short prompt on a small layer: latency.
        _case("attn_200", "attn", "0", "200", Hkv=2),
        # An ordinary prompt.
        _case("attn_8k", "attn", "0", "8192"),
        # The prompt of the 32K configuration.
        _case("attn_32k", "attn", "0", "32003"),
        # A chunk of a long prompt, behind what its earlier chunks left.
        _case("attn_chunk", "attn", "120001", "512"),
        # A batch of prompts of very different lengths, eight query heads to a KV head.
        _case("attn_batch", "attn", "0,0,0,0,0,0,0,0,0,0", "4001,33,1,1025,2500,700,129,64,6007,317", Hkv=4, G=8),
        # A few tokens for each of several long contexts (drafted tokens that are checked in one pass).
        _case("attn_few", "attn", "20011,47777,65537,90001", "5,1,8,3"),
        # The decode token of one small layer with one satellite: latency.
        _case("append_1", "append", "4096", "1", Hkv=2, n_full=1, n_sat=1, rot=128, pairs="half", scaling="none", norm=True, type="bf16", theta=10000.0),
        # The decode tokens of a large serving batch.
        _case("append_64", "append", ",".join(str(2048 + 517 * i) for i in range(64)), ",".join(["1"] * 64), n_full=2, n_sat=0, rot=128, pairs="interleaved",
              scaling="bands", norm=True, type="bf16", theta=500000.0),
    ]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rope", "attn", "attn", "attn", "append"])
    Hkv, G = rng.choice([1, 2, 4, 8, 8]), rng.choice([1, 2, 4, 4, 8])
    if kind == "attn":
        flops = math.inf
        while flops > 8.3e12:
            B = rng.choice([1, 1, 2, 5, 12])
            count = [_logint(rng, 1, 16384) for _ in range(B)]
            first = [rng.choice([0, 0, _logint(rng, 1, 131072)]) for _ in range(B)]
            flops = sum(512 * Hkv * G * n * (f + (n + 1) / 2) for f, n in zip(first, count))
        return _case(None, "attn", ",".join(map(str, first)), ",".join(map(str, count)), Hkv=Hkv, G=G)
    more = dict(rot=rng.choice([128, 128, 64, 32, 96]), pairs=rng.choice(["half", "interleaved"]), scaling=rng.choice(["none", "linear", "base", "bands"]),
                norm=rng.choice([True, False]), type=rng.choice(["bf16", "bf16", "f32"]), theta=rng.choice([10000.0, 500000.0]))
    if kind == "rope":
        B = rng.choice([1, 2, 4, 9])
        count = [_logint(rng, 1, 8192) for _ in range(B)]
        first = [rng.choice([0, _logint(rng, 1, 131072)]) for _ in range(B)]
        return _case(None, "rope", ",".join(map(str, first)), ",".join(map(str, count)), Hkv=Hkv, G=G, **more)
    B = _logint(rng, 1, 64)
    first = [_logint(rng, 300, 32768) for _ in range(B)]
    return _case(None, "append", ",".join(map(str, first)), ",".join(["1"] * B), Hkv=Hkv, G=G, n_full=rng.randint(1, max(1, Hkv // 2)), n_sat=0, **more)


def _ints(s):
    return [int(x) for x in s.split(",")]


# ---- what a user's program holds ------------------------------------------------------------------------------------------------------

SINK, RECENT, SLOTS = 64, 128, 256       # of a compressed head of the append cases


def _room(c):
    """Rows of every sequence's K and V blocks in the prompt's buffer: a multiple of 64 behind the last token."""
    return [(f + n + 63) // 64 * 64 for f, n in zip(_ints(c["first"]), _ints(c["count"]))]


def _offsets(c):
    """Element offsets of the heads' K and V blocks in the prompt's buffer, sequence by sequence, and its size."""
    k_off, v_off, at = [], [], 0
    for rows in _room(c):
        for _ in range(c["Hkv"]):
            k_off.append(at)
            v_off.append(at + rows * D)
            at += 2 * rows * D
    return k_off, v_off, at


def _cache(c):
    """The append cases' cache: (role, offset of K, offset of V, tier offset) of every head; elements of cache and host tier."""
    heads, at, tier = [], 0, 0
    for n in _ints(c["first"]):
        for h in range(c["Hkv"]):
            role = 0 if h < c["n_full"] else 1 if h < c["n_full"] + c["n_sat"] else 2
            rows = n + GROW if role == 0 else SLOTS
            heads.append((role, at, at + rows * D, tier))
            at += 2 * rows * D
            if role == 1:
                tier += (n + GROW) * 2 * D
    return heads, at, tier


def _rope_inputs(c, g, T):
    """What the projections leave, q, k and v side by side in one row a token, and the weights of the two norms."""
    Hq, Hkv = c["Hkv"] * c["G"], c["Hkv"]
    x = torch.randn((T, Hq + 2 * Hkv, D), generator=g, device=DEV)
    x *= torch.exp(0.5 * torch.randn((Hq + 2 * Hkv, D), generator=g, device=DEV))          # channels differ in size
    w = [1 + 0.2 * torch.randn((D,), generator=g, device=DEV) for _ in range(2)] if c["norm"] else [None, None]
    return x.to(torch.bfloat16 if c["type"] == "bf16" else torch.float32), w[0], w[1]


def _context(c, max_ctx):
    from paper_2601_13684_amd import binding as hc
    cfg = hc.hc_config(B=len(_ints(c["first"])), Hq=c["Hkv"] * c["G"], Hkv=c["Hkv"], D=D, max_ctx=(max(max_ctx, SLOTS) + 63) // 64 * 64, max_k=SLOTS, window=1,
                       metric=0, tau_num=4, tau_den=5, agg=0, window_mode=0)
    return Handle(hc.hc_create(cfg), hc.hc_destroy)



class Handle:
    """A library object that lives as long as the state does."""

    def __init__(self, value, close, after=None):
        self.value, self.close, self.after = value, close, after

    def __del__(self):
        torch.cuda.synchronize()
        self.close(self.value)


def _rope(s):
    """The model's rotation and norms, as the library takes them."""
    from paper_2601_13684_amd import binding as hc
    c = s["c"]
    kinds = dict(linear=hc.HC_ROPE_LINEAR, base=hc.HC_ROPE_BASE, bands=hc.HC_ROPE_BANDS)
    scaling = hc.hc_rope_scaling(kind=kinds[c["scaling"]], **SCALING[c["scaling"]]) if c["scaling"] != "none" else None
    return hc.hc_rope_init(hc.HC_ROPE_HALF if c["pairs"] == "half" else hc.HC_ROPE_INTERLEAVED, c["rot"], c["theta"], scaling,
                           q_norm=s["q_norm"], k_norm=s["k_norm"], eps=EPS)


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    first, count = _ints(c["first"]), _ints(c["count"])
    B, Hkv, G = len(first), c["Hkv"], c["G"]
    Hq, T = Hkv * G, sum(count)
    s = dict(c=c, first=first, count=count)
    if c["kind"] == "append":
        heads, size, tier = _cache(c)
        s["x"], s["q_norm"], s["k_norm"] = _rope_inputs(c, g, B)
        # (appending reads nothing of the cache: of zeros, so that what is written is what counts)
        s["arena"] = torch.zeros((size,), dtype=torch.bfloat16, device=DEV)
        s["tier"] = torch.zeros((tier,), dtype=torch.bfloat16, pin_memory=True) if tier else None
        s["q_out"] = torch.zeros((B, Hq, D), dtype=torch.bfloat16, device=DEV)
        if own:
            from paper_2601_13684_amd import binding as hc
            s["ctx"], s["rope"] = _context(c, max(first) + GROW), _rope(s)
            descs = [hc.hc_head_desc(k_off=k, v_off=v, tier_off=t, ctx=first[i // Hkv], len=first[i // Hkv] if role == 0 else SLOTS, role=role,
                                     rep=0 if role == 1 else -1, sink=0 if role == 0 else SINK, recent=0 if role == 0 else RECENT, k_mon=0,
                                     cap=first[i // Hkv] + GROW if role < 2 else 0) for i, (role, k, v, t) in enumerate(heads)]
            s["layer"] = Handle(hc.hc_layer_create(s["ctx"].value, descs), hc.hc_layer_destroy, s["ctx"])
        else:
            at = lambda j: torch.tensor([h[j] // D for h in heads], device=DEV)  # noqa: E731
            s["pos"] = torch.tensor(first, device=DEV)
            s["first_pos"] = s["pos"].clone()
            s["k_row"], s["v_row"] = at(1).view(B, Hkv), at(2).view(B, Hkv)
            s["full"] = torch.tensor([h[0] == 0 for h in heads], device=DEV).view(B, Hkv)
            s["sat"] = [(i, h[3] // D) for i, h in enumerate(heads) if h[0] == 1]
            s["steps"] = 0
        return s
    k_off, v_off, size = _offsets(c)
    s["k_off"], s["v_off"] = k_off, v_off
    if c["kind"] == "rope":
        s["x"], s["q_norm"], s["k_norm"] = _rope_inputs(c, g, T)
        s["kv"] = torch.zeros((size,), dtype=torch.bfloat16, device=DEV)
        s["q_out"] = torch.zeros((T, Hq, D), dtype=torch.bfloat16, device=DEV)
        if not own:
            s["pos"] = torch.cat([torch.arange(f, f + n, device=DEV) for f, n in zip(first, count)])
            seq = torch.repeat_interleave(torch.arange(B, device=DEV), torch.tensor(count, device=DEV))
            rows = lambda off: (torch.tensor(off, device=DEV) // D).view(B, Hkv)[seq] + s["pos"][:, None]  # noqa: E731
            s["k_row"], s["v_row"] = rows(k_off), rows(v_off)
    else:
        # queries and keys as rotation leaves them: logits of standard deviation 1.5, a first position that draws attention
        # wherever one looks from, and one position in 50 that draws more than the rest
        s["q"] = (1.5 * torch.randn((T, Hq, D), generator=g, device=DEV) + 0.3).to(torch.bfloat16)
        kv = torch.randn((size // D, D), generator=g, device=DEV)
        u = torch.ones((D,), device=DEV)
        k_rows = torch.tensor(k_off, device=DEV) // D
        heavy = torch.rand((size // D,), generator=g, device=DEV) < 0.02
        kv[heavy] += 0.4 * u
        kv[k_rows] += 0.8 * u
        s["kv"] = kv.to(torch.bfloat16).view(-1)
        if own:
            s["out"] = torch.zeros((T, Hq, D), dtype=torch.bfloat16, device=DEV)
            s["lse"] = torch.zeros((T, Hq), dtype=torch.float32, device=DEV)
    if own:
        from paper_2601_13684_amd import binding as hc
        s["ctx"] = _context(c, max(_room(c)))
        if c["kind"] == "rope":
            s["rope"] = _rope(s)
        else:
            s["work"] = torch.zeros((hc.hc_prefill_attn_work_bytes(s["ctx"].value),), dtype=torch.uint8, device=DEV)
    return s


# ---- one pass -------------------------------------------------------------------------------------------------------------------------

def run(state):
    if own:
        return _run_own(state)
    return {"rope": _plain_rope, "attn": _plain_attn, "append": _plain_append}[state["c"]["kind"]](state)


def _run_own(s):
    from paper_2601_13684_amd import binding as hc
    c = s["c"]
    if c["kind"] == "attn":
        hc.hc_prefill_attn(s["ctx"].value, s["q"], s["kv"], s["k_off"], s["v_off"], s["first"], s["count"], s["out"], s["lse"], s["work"], s["work"].numel())
        return s["out"], s["lse"]
    Hkv, Hq, x = c["Hkv"], c["Hkv"] * c["G"], s["x"]
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    if c["kind"] == "rope":
        hc.hc_prefill_rope(s["ctx"].value, s["rope"], q, k, v, s["first"], s["count"], s["q_out"], s["kv"], s["k_off"], s["v_off"])
        return s["q_out"], s["kv"]
    hc.hc_append_rope(s["ctx"].value, s["layer"].value, s["rope"], q, k, v, s["q_out"], s["arena"], s["tier"])
    return (s["q_out"], s["arena"]) if s["tier"] is None else (s["q_out"], s["arena"], s["tier"])


def _frequencies(c):
    """Radians a position, 64 bits."""
    i = torch.arange(0, c["rot"], 2, dtype=torch.float64, device=DEV) / c["rot"]
    p = SCALING.get(c["scaling"])
    if c["scaling"] == "base":
        return (c["theta"] * p["factor"] ** (c["rot"] / (c["rot"] - 2))) ** -i
    f = c["theta"] ** -i
    if c["scaling"] == "linear":
        return f / p["factor"]
    if c["scaling"] == "bands":
        keep = ((p["original"] * f / (2 * math.pi) - p["low"]) / (p["high"] - p["low"])).clamp(0, 1)
        return f * keep + f / p["factor"] * (1 - keep)
    return f


def _turn(c, x, weight, cos, sin):
    """Norm and rotation of x [T, heads, 128], 32 bits."""
    if weight is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight
    r = c["rot"]
    if c["pairs"] == "half":
        a, b = x[..., :r // 2], x[..., r // 2:r]
        return torch.cat([a * cos - b * sin, b * cos + a * sin, x[..., r:]], -1).to(torch.bfloat16)
    a, b = x[..., 0:r:2], x[..., 1:r:2]
    return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2), x[..., r:]], -1).to(torch.bfloat16)


def _turned(s):
    """q and k turned, v as it is, of the tokens at the positions s["pos"]."""
    c = s["c"]
    Hkv, Hq = c["Hkv"], c["Hkv"] * c["G"]
    angle = s["pos"].double()[:, None, None] * _frequencies(c)
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    x = s["x"].float()
    return _turn(c, x[:, :Hq], s["q_norm"], cos, sin), _turn(c, x[:, Hq:Hq + Hkv], s["k_norm"], cos, sin), x[:, Hq + Hkv:].to(torch.bfloat16)


def _plain_rope(s):
    q, k, v = _turned(s)
    rows = s["kv"].view(-1, D)
    rows[s["k_row"]] = k
    rows[s["v_row"]] = v
    s["q_out"].copy_(q)
    return s["q_out"], s["kv"]


def _plain_append(s):
    c = s["c"]
    q, k, v = _turned(s)
    pos = s["pos"][:, None]
    slot = torch.where(s["full"], pos, SINK + (pos - s["first_pos"][:, None]) % RECENT)
    rows = s["arena"].view(-1, D)
    rows[s["k_row"] + slot] = k
    rows[s["v_row"] + slot] = v
    for i, row in s["sat"]:              # the satellites' rows go to host memory too
        to = s["tier"].view(-1, D)[row + 2 * (s["first"][i // c["Hkv"]] + s["steps"]):][:2]
        to.copy_(torch.stack([k.view(-1, D)[i], v.view(-1, D)[i]]), non_blocking=True)
    s["pos"] += 1
    s["steps"] += 1
    s["q_out"].copy_(q)
    return (s["q_out"], s["arena"]) if s["tier"] is None else (s["q_out"], s["arena"], s["tier"])


def _blocks(c, most):
    """(sequence, first token, tokens, rows of keys that its last token sees) of pieces of the queries whose logits are at most `most` values."""
    row = 0
    for f, n in zip(_ints(c["first"]), _ints(c["count"])):
        step = max(1, int(most // (c["Hkv"] * c["G"] * (f + n))))
        for i in range(0, n, step):
            yield row + i, min(step, n - i), f + i
        row += n


def _plain_attn(s):
    c = s["c"]
    Hkv, G = c["Hkv"], c["G"]
    T = sum(s["count"])
    out = torch.empty((T, Hkv, G, D), dtype=torch.bfloat16, device=DEV)
    lse = torch.empty((T, Hkv, G), dtype=torch.float32, device=DEV)
    q = s["q"].view(T, Hkv, G, D).permute(1, 0, 2, 3).float() / math.sqrt(D)
    ends, b, row = [sum(s["count"][:i + 1]) for i in range(len(s["count"]))], -1, 0
    rows = _room(c)
    for at, n, p in _blocks(c, 2 ** 30):
        if b < 0 or at >= ends[b]:       # the next sequence that has tokens: its keys and values
            b = next(i for i, e in enumerate(ends) if at < e)
            kv = s["kv"][s["k_off"][b * Hkv]:][:2 * Hkv * rows[b] * D].view(Hkv, 2, rows[b], D).float()
            k, v = kv[:, 0].transpose(1, 2).contiguous(), kv[:, 1].contiguous()
        see = p + n                      # positions that the block's last token sees
        x = torch.bmm(q[:, at:at + n].reshape(Hkv, n * G, D), k[:, :, :see].contiguous()).view(Hkv, n, G, see)
        hidden = torch.arange(see, device=DEV) > torch.arange(p, p + n, device=DEV)[:, None]
        x.masked_fill_(hidden[:, None, :], -math.inf)
        top = x.amax(-1, keepdim=True)
        x.sub_(top).exp_()
        total = x.sum(-1, keepdim=True)
        o = torch.bmm(x.view(Hkv, n * G, see), v[:, :see].contiguous()).view(Hkv, n, G, D) / total
        out[at:at + n] = o.permute(1, 0, 2, 3).to(torch.bfloat16)
        lse[at:at + n] = (top + total.log())[..., 0].permute(1, 0, 2)
    return out.view(T, Hkv * G, D), lse.view(T, Hkv * G)


# ---- the same in 64 bits --------------------------------------------------------------------------------------------------------------

def exact(case, seed):
    c = case
    s = prepare(c, seed)
    if c["kind"] == "attn":
        return _exact_attn(s)
    Hkv, Hq = c["Hkv"], c["Hkv"] * c["G"]
    first, count = s["first"], s["count"]
    x = s["x"].double()
    pos = torch.tensor([f + i for f, n in zip(first, count) for i in range(n)], dtype=torch.float64, device=DEV)
    # a pair is a complex number, turned by exp(i angle)
    half = torch.arange(c["rot"] // 2, dtype=torch.float64, device=DEV)
    p = SCALING.get(c["scaling"], {})
    base = c["theta"] * (p["factor"] ** (c["rot"] / (c["rot"] - 2.0)) if c["scaling"] == "base" else 1.0)
    f = torch.exp(-2 * half / c["rot"] * math.log(base))
    if c["scaling"] == "linear":
        f = f / p["factor"]
    if c["scaling"] == "bands":
        turns = p["original"] * f / (2 * math.pi)          # full turns inside the original context
        part = (turns - p["low"]) / (p["high"] - p["low"])
        f = torch.where(turns < p["low"], f / p["factor"], torch.where(turns > p["high"], f, (1 - part) * f / p["factor"] + part * f))
    e = torch.polar(torch.ones_like(f * pos[:, None]), f * pos[:, None])[:, None]
    i = torch.arange(c["rot"] // 2, device=DEV)
    one, two = (i, i + c["rot"] // 2) if c["pairs"] == "half" else (2 * i, 2 * i + 1)
    done = []
    for y, w in ((x[:, :Hq], s["q_norm"]), (x[:, Hq:Hq + Hkv], s["k_norm"])):
        y = y.clone()
        if w is not None:
            y = y / torch.sqrt((y * y).sum(-1, keepdim=True) / D + EPS) * w.double()
        z = torch.complex(y[..., one], y[..., two]) * e
        y[..., one], y[..., two] = z.real, z.imag
        done.append(y)
    q, k, v = done[0], done[1], x[:, Hq + Hkv:]
    if c["kind"] == "rope":
        kv = torch.zeros((s["kv"].numel() // D, D), dtype=torch.float64, device=DEV)
        t = 0
        for b, (f0, n) in enumerate(zip(first, count)):
            for h in range(Hkv):
                at_k, at_v = s["k_off"][b * Hkv + h] // D + f0, s["v_off"][b * Hkv + h] // D + f0
                kv[at_k:at_k + n], kv[at_v:at_v + n] = k[t:t + n, h], v[t:t + n, h]
            t += n
        return q, kv.view(-1)
    heads, size, tier = _cache(c)
    arena = torch.zeros((size // D, D), dtype=torch.float64, device=DEV)
    host = torch.zeros((tier // D, D), dtype=torch.float64)
    for j, (role, k_off, v_off, t_off) in enumerate(heads):
        b, h = divmod(j, Hkv)
        slot = first[b] if role == 0 else SINK             # the first token behind the prompt takes the oldest recent slot
        arena[k_off // D + slot], arena[v_off // D + slot] = k[b, h], v[b, h]
        if role == 1:
            host[t_off // D + 2 * first[b]], host[t_off // D + 2 * first[b] + 1] = k[b, h].cpu(), v[b, h].cpu()
    return (q, arena.view(-1)) if s["tier"] is None else (q, arena.view(-1), host.view(-1))


def _exact_attn(s):
    c = s["c"]
    Hkv, G = c["Hkv"], c["G"]
    T = sum(s["count"])
    out = torch.zeros((T, Hkv * G, D), dtype=torch.float64, device=DEV)
    lse = torch.zeros((T, Hkv * G), dtype=torch.float64, device=DEV)
    t = 0
    for b, (f, n) in enumerate(zip(s["first"], s["count"])):
        for h in range(Hkv):
            k, v = (s["kv"][off[b * Hkv + h]:off[b * Hkv + h] + (f + n) * D].view(f + n, D).double() for off in (s["k_off"], s["v_off"]))
            step = max(1, 2 ** 28 // ((f + n) * G))
            for i in range(0, n, step):
                m = min(step, n - i)
                x = s["q"][t + i:t + i + m, h * G:(h + 1) * G].double().reshape(m * G, D) @ k[:f + i + m].t().contiguous() * D ** -0.5
                p = torch.arange(f + i, f + i + m, device=DEV).repeat_interleave(G)
                x = torch.where(torch.arange(f + i + m, device=DEV)[None] <= p[:, None], x, torch.full((), -math.inf, dtype=torch.float64, device=DEV))
                l = torch.logsumexp(x, -1)
                out[t + i:t + i + m, h * G:(h + 1) * G] = (torch.exp(x - l[:, None]) @ v[:f + i + m]).view(m, G, D)
                lse[t + i:t + i + m, h * G:(h + 1) * G] = l.view(m, G)
        t += n
    return out, lse


def work(case):
    c = case
    first, count = _ints(c["first"]), _ints(c["count"])
    Hkv, Hq, T = c["Hkv"], c["Hkv"] * c["G"], sum(count)
    if c["kind"] == "attn":
        pairs = sum(n * f + n * (n + 1) // 2 for f, n in zip(first, count))
        return dict(bytes=T * Hq * (2 * D * 2 + 4) + sum(f + n for f, n in zip(first, count)) * Hkv * 2 * D * 2, flops=4 * D * Hq * pairs)
    size = 2 if c["type"] == "bf16" else 4
    values = T * (Hq + 2 * Hkv) * D
    return dict(bytes=values * (size + 2) + (T * c["n_sat"] * 2 * D * 2 if c["kind"] == "append" else 0), flops=T * (Hq + Hkv) * (3 * c["rot"] + (4 * D if c["norm"] else 0)))
