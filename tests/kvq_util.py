"""Plain 64-bit forms of the operators of the cache held in 4 bits, written from the format's and the operators' definitions."""
import math

import torch

from paper_2601_13684_amd import binding as hc

DEV = "cuda:0"
D = 128
SIZES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def context(B, Hkv, G, max_ctx):
    return hc.hc_create(hc.hc_config(B=B, Hq=Hkv * G, Hkv=Hkv, D=D, max_ctx=(max_ctx + 63) // 64 * 64, max_k=8, window=1, metric=0, tau_num=1, tau_den=2,
                                     agg=0, window_mode=0))


class Cache:
    """A table over `caps` rows a head with gaps between the blocks and between the rows' tables, and buffers of it filled with a pattern."""

    def __init__(self, ctx, caps, rows=None, pos=None, budget=None, sink=0, recent=0, gap=64, dev=DEV):
        self.ctx, self.caps, self.heads = ctx, list(caps), []
        at, row = gap, 3 if gap else 0
        for i, cap in enumerate(caps):
            self.heads.append(hc.hc_kvq_head(off=at, row_off=row, cap=cap, budget=cap if budget is None else budget[i], sink=sink, recent=recent))
            at += 136 * cap + gap
            row += cap + (5 if gap else 0)
        self.bytes, self.rows = at, row
        self.kvq = hc.hc_kvq_create(ctx, self.heads)
        self.arena = torch.full((at,), 0xA5, dtype=torch.uint8, device=dev)
        n = [0] * len(caps) if rows is None else list(rows)
        self.state = torch.tensor(list(zip(n, n if pos is None else pos)), dtype=torch.int32, device=dev).view(-1, 2)
        self.acc = torch.full((row,), 7.5, device=dev)

    def blocks(self, i, v):
        """Views of head i's codes [cap, 64] and scales [cap, 4] of K (v: of V)."""
        cap, off = self.caps[i], self.heads[i].off + 68 * self.caps[i] * v
        return self.arena[off:off + 64 * cap].view(cap, 64), self.arena[off + 64 * cap:off + 68 * cap].view(cap, 4)

    def put(self, i, v, row, x):
        """Rows x (bf16) into the buffers, by the format's definition."""
        c, s = encode(x)
        codes, scales = self.blocks(i, v)
        codes[row:row + len(x)], scales[row:row + len(x)] = c, s

    def held(self, i, v, n=None):
        codes, scales = self.blocks(i, v)
        return decode(codes[:n], scales[:n])

    def work(self):
        return torch.zeros((hc.hc_kvq_work_bytes(self.ctx, self.kvq),), dtype=torch.uint8, device=self.arena.device)

    def close(self):
        torch.cuda.synchronize()
        hc.hc_kvq_destroy(self.kvq)


def units(x):
    """The scale bytes of rows x [n, 128]: the smallest s >= 2 with every |x| <= 7 * 2^(s - 127), 255 where one is not finite."""
    top = x.double().abs().view(-1, 4, 32).amax(-1)
    s = torch.full(top.shape, 2, dtype=torch.int32, device=x.device)
    for k in range(2, 254):
        s += (top > 7 * 2.0 ** (k - 127)).int() * (s == k).int()
    return torch.where(torch.isfinite(x.double()).view(-1, 4, 32).all(-1), s, 255).to(torch.uint8)


def encode(x):
    """Codes [n, 64] and scales [n, 4] of rows x, by trying every code: the nearest, of two equally near the even one."""
    s = units(x)
    m = x.double().view(-1, 4, 32) * 2.0 ** (127 - s.double())[..., None]
    sizes = torch.tensor(SIZES, dtype=torch.float64, device=x.device)
    far = (m.abs()[..., None] - sizes).abs()
    far = torch.where(torch.arange(8, device=x.device) % 2 == 0, far, far * (1 + 1e-12))        # (ties to even)
    code = torch.where((s == 255)[..., None], 0, far.argmin(-1) + 8 * torch.signbit(x.double().view(-1, 4, 32)).long()).view(-1, 64, 2)
    return (code[..., 0] + 16 * code[..., 1]).to(torch.uint8), s


def decode(codes, scales):
    c = torch.stack([codes & 15, codes >> 4], -1).long().flatten(-2)
    size = torch.tensor(SIZES + tuple(-x for x in SIZES), dtype=torch.float64, device=codes.device)[c]
    unit = torch.where(scales == 255, math.nan, 2.0 ** (scales.double() - 127))
    return size * unit.repeat_interleave(32, dim=-1)


def rows_of(n, seed, kind="plain", dev=DEV):
    """n rows of bf16; kinds that meet the format's borders."""
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    x = torch.randn((n, D), generator=g, device=dev) * torch.exp(0.7 * torch.randn((D,), generator=g, device=dev))
    if kind == "borders":        # values at the borders between codes, and groups whose largest is at the border between scales
        m = torch.tensor([0.0, 0.25, 0.5, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, 7.03125, 3.515625, 0.24951171875], device=dev)
        x = m[torch.randint(0, len(m), (n, D), generator=g, device=dev)] * (1 - 2 * torch.randint(0, 2, (n, D), generator=g, device=dev))
        x = x * 2.0 ** torch.randint(-20, 20, (n, 4), generator=g, device=dev).repeat_interleave(32, dim=1)
    if kind == "tiny":           # about the smallest scale, subnormal numbers among them
        x = x * 2.0 ** torch.randint(-134, -122, (n, 4), generator=g, device=dev).double().repeat_interleave(32, dim=1)
    if kind == "huge":
        x = x.clamp(-3, 3) * 2.0 ** 125
    x = x.to(torch.bfloat16)
    if kind == "odd":            # zeros of both signs, whole groups of them, infinities and NaNs
        x[torch.rand((n, D), generator=g, device=dev) < 0.2] = 0.0
        x[torch.rand((n, D), generator=g, device=dev) < 0.1] = -0.0
        x.view(n, 4, 32)[torch.rand((n, 4), generator=g, device=dev) < 0.2] = 0.0
        for bad in (math.inf, -math.inf, math.nan):
            x[torch.rand((n, D), generator=g, device=dev) < 0.003] = bad
    return x


def attention(q, K, V):
    """out [G, 128], lse [G], weights [G, n] and sum p |v| of q [G, 128] over rows K, V (64 bits)."""
    s = q.double() @ K.t().contiguous() / math.sqrt(D)
    lse = torch.logsumexp(s, -1)
    p = torch.exp(s - lse[:, None])
    return p @ V, lse, p, p @ V.abs()


def check_attention(cache, q, G, out, lse, acc=None, acc_before=None, decay=1.0, where=""):
    """The products are exact in their factors; sums are 32-bit.  A logit sums 128 products in some order: 128 roundings of 2^-24 of sum |q k| / sqrt(128) at
    most, two more of the scaled value, and the reference's: below e = 2^-24 (130 sum |q k| / sqrt(128) + 4 |s|).  A weight is then off by e, by the
    exponential's 2^-22 and by what the logits' largest is off, twice in a ratio; the sums over n rows by (n / 8 + 64) 2^-24 of sum p |v|, since a sum is
    made of parallel ones of at most n / 32 terms each (four lanes' groups of 8 rows at a time): taken as n / 8."""
    heads = len(cache.caps)
    rows = cache.state[:, 0].tolist()
    q, out, lse = q.view(heads, G, D), out.view(heads, G, D), lse.view(heads, G)
    for i in range(heads):
        n = rows[i]
        if n == 0:
            assert (out[i] == 0).all() and (lse[i] == -math.inf).all(), (where, i)
            continue
        K, V = cache.held(i, 0, n), cache.held(i, 1, n)
        o, l, p, pv = attention(q[i], K, V)
        size = (q[i].double().abs() @ K.abs().t().contiguous()).amax(-1) / math.sqrt(D)
        e = 2.0 ** -24 * (130 * size + 4 * l.abs()) + 2.0 ** -22
        tol = (2 * e + (n / 8 + 64) * 2.0 ** -24)[:, None]
        err = (out[i].double() - o).abs()
        assert (err <= tol * pv + 1e-38).all(), (where, i, n, float((err / (tol * pv + 1e-38)).max()))
        assert ((lse[i].double() - l).abs() <= tol[:, 0] + 2.0 ** -22 * l.abs()).all(), (where, i, n, "lse")
        if acc is not None:
            r = cache.heads[i].row_off
            want = acc_before[r:r + n].double() * decay + p.mean(0)
            err = (acc[r:r + n].double() - want).abs()
            assert (err <= (tol * p).mean(0) + 2.0 ** -22 * want).all(), (where, i, n, "acc", float(err.max()))


def survivors(n, budget, sink, recent, acc):
    """Which of n rows stay, by sorting."""
    if n <= budget:
        return list(range(n))
    score = [(-math.inf if a != a else a) for a in acc[:n].tolist()]
    nan = [a != a for a in acc[:n].tolist()]
    between = sorted(range(sink, n - recent), key=lambda r: (nan[r], -score[r], r))[:budget - sink - recent]
    return list(range(sink)) + sorted(between) + list(range(n - recent, n))
