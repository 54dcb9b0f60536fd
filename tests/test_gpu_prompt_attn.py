"""hc_prefill_attn against the 64-bit form.  Run with `-m gpu` on an MI355X."""
import math

import pytest
import torch

from paper_2601_13684_amd import binding as hc

import prompt_util as P

pytestmark = pytest.mark.gpu
DEV, D = P.DEV, P.D


class Call:
    def __init__(self, first, count, Hkv, G, seed=0, gap=0, spread=1.0):
        print("prompt attention", first, count, Hkv, G, flush=True)
        self.first, self.count, self.Hkv, self.G = first, count, Hkv, G
        g = torch.Generator(device=DEV)
        g.manual_seed(seed + 1)
        self.T = sum(count)
        room = [f + n for f, n in zip(first, count)]
        self.k_off, self.v_off, size = P.blocks(room, Hkv, gap)
        self.kv = torch.randn((size,), generator=g, device=DEV).to(torch.bfloat16)
        self.q = (spread * torch.randn((self.T, Hkv * G, D), generator=g, device=DEV)).to(torch.bfloat16)
        self.out = torch.full((self.T + 1, Hkv * G, D), 7.0, dtype=torch.bfloat16, device=DEV)
        self.lse = torch.full((self.T + 1, Hkv * G), 7.0, device=DEV)
        self.ctx = P.context(len(first), Hkv, G, max(room + [1]))
        self.work = torch.empty((hc.hc_prefill_attn_work_bytes(self.ctx),), dtype=torch.uint8, device=DEV)
        self.work.fill_(255)                     # NaN in every place

    def run(self, lse=True, stream=None):
        hc.hc_prefill_attn(self.ctx, self.q, self.kv, self.k_off, self.v_off, self.first, self.count, self.out, self.lse if lse else None, self.work,
                           self.work.numel(), stream)

    def want(self):
        return P.attention(self.q, self.kv, self.k_off, self.v_off, self.first, self.count, self.Hkv, self.G)

    def check(self, where=""):
        torch.cuda.synchronize()
        P.check_attention(self.out[:self.T], self.lse[:self.T], self.want(), where)
        assert (self.out[self.T:] == 7).all() and (self.lse[self.T:] == 7).all()

    def close(self):
        hc.hc_destroy(self.ctx)


ONE = [(0, 1), (0, 2), (0, 15), (0, 31), (0, 33), (0, 63), (0, 64), (0, 65), (0, 127), (0, 129), (0, 257), (63, 1), (64, 1), (62, 3), (1, 64), (1000, 17),
       (255, 1), (256, 1), (257, 2), (5000, 1), (5000, 130), (300, 1000)]


@pytest.mark.parametrize("G", [1, 2, 4, 8])
@pytest.mark.parametrize("first,count", ONE)
def test_one_sequence(first, count, G):
    c = Call([first], [count], 2, G, seed=count)
    c.run()
    c.check()
    c.close()


@pytest.mark.parametrize("first,count,Hkv,G", [
    ([0, 0, 0], [5, 0, 300], 3, 4),                              # one that brings nothing
    ([0, 700, 64], [0, 1, 64], 1, 8),
    ([17 * i for i in range(70)], [1 + i % 3 for i in range(70)], 2, 4),          # more sequences than a launch takes
    ([40 * i for i in range(40)], [(i * i) % 50 for i in range(40)], 8, 2),       # more heads than a launch takes
    ([0, 9000], [2000, 1], 8, 4),                                # whole tiles of one beside a long axis of the other
    ([0], [2500], 16, 1),
    ([100, 0], [40, 77], 128, 1),                                # as many heads as a call takes
    ([12000, 20011, 47777], [5, 1, 8], 8, 4),
    ([0, 0], [4097, 63], 8, 8),
])
def test_packed(first, count, Hkv, G):
    c = Call(first, count, Hkv, G, gap=8)
    c.run()
    c.check()
    c.close()


@pytest.mark.parametrize("first,count,Hkv,G", [
    ([0], [8777], 1, 1), ([0], [4100], 2, 1), ([300], [6001], 1, 2),           # a prompt in pieces: its tiles have different numbers of them
    ([60001], [52], 1, 8), ([62133, 0], [42, 14], 2, 4), ([50001], [150], 4, 1), ([33000], [301], 3, 4),      # a chunk: pieces of one head alternate
    ([20000, 3000, 0], [1, 5000, 700], 1, 4),
])
def test_pieces_of_few_heads(first, count, Hkv, G):
    c = Call(first, count, Hkv, G)
    c.run()
    c.check()
    c.close()


def test_nothing_to_do():
    c = Call([5, 0], [0, 0], 2, 4)
    c.run()
    torch.cuda.synchronize()
    assert (c.out == 7).all() and (c.lse == 7).all()
    c.close()


@pytest.mark.parametrize("first,count", [(0, 300), (3000, 3), (131072, 9)])
def test_peaked_logits_and_no_lse(first, count):
    """Logits of standard deviation 6: the reference moves often and most weights are nothing."""
    c = Call([first], [count], 2, 4, spread=6.0)
    c.run()
    c.check()
    out = c.out.clone()
    c.out.fill_(7)
    c.run(lse=False)
    torch.cuda.synchronize()
    assert torch.equal(c.out, out)
    c.close()


def test_growing_logits():
    """Every key is larger than all before it: the reference moves at every step, by up to hundreds of binary orders."""
    c = Call([0], [700], 1, 4)
    up = torch.linspace(-60, 60, 700, device=DEV)
    c.kv[c.k_off[0]:c.k_off[0] + 700 * D] = (up[:, None] * torch.ones(D, device=DEV)).to(torch.bfloat16).view(-1)
    c.q.fill_(1.0)
    c.run()
    c.check()
    c.close()


# one tile of rows, tiles with and without whole ones in front, pieces of the keys, both tile heights, one row
SHAPES = [([0], [40], 2, 4), ([0], [700], 2, 1), ([0], [2500], 8, 4), ([9000], [2], 2, 8), ([9000], [64], 8, 4), ([40000], [400], 8, 1), ([20000, 0, 300], [1, 1500, 70], 2, 2)]


def per_key(c, offsets, value):
    """value(position) of every key into the rows at offsets."""
    for b, (f, n) in enumerate(zip(c.first, c.count)):
        for h in range(c.Hkv):
            o = offsets[b * c.Hkv + h]
            rows = c.kv[o:o + (f + n) * D].view(f + n, D)
            rows.copy_(value(torch.arange(f + n, device=DEV, dtype=torch.float64), rows))


@pytest.mark.parametrize("first,count,Hkv,G", SHAPES)
@pytest.mark.parametrize("rise", [-0.75, 0.25, 4.0])
def test_logits_that_rise_with_the_position(first, count, Hkv, G, rise):
    """By `rise` from key to key (up to 2^17 in all): far beyond what weights against the first keys' largest could hold.  q . K = position * rise * sqrt(128)
    but for what the other elements bring, each product exact: bf16 steps of the position make two keys of the same logit, as in the oracle."""
    c = Call(first, count, Hkv, G, seed=5)
    c.q[..., 1:] = 0
    c.q[..., 0] = 1
    per_key(c, c.k_off, lambda at, rows: torch.cat([(at * (rise * math.sqrt(D)))[:, None], rows[:, 1:].double()], 1).to(torch.bfloat16))
    c.run()
    torch.cuda.synchronize()
    o, lse, pv, p2 = c.want()
    # one product a logit: a weight is off by the rounding of t = s log2(e) / sqrt(128) and of t - ref, 2^-23 |t|, below 2^-4.7 for |t| up to 2^18.3; twice in a ratio.
    # The keys that count have t within a few binary orders of the row's largest, and errors of the factor are common to all of them
    # where their logits are equal; what is left is held to the 2^-10 that check_attention gives, plus 2^-22 |s| for unequal ones.
    tol = 2.0 ** -8 * (pv + o.abs()) + (2.0 ** -10 + 2.0 ** -22 * lse.abs())[..., None] * pv
    err = (c.out[:c.T].double() - o).abs()
    assert (err <= tol).all(), float((err - tol).max())
    assert ((c.lse[:c.T].double() - lse).abs() <= 1e-4 + 1e-6 * lse.abs()).all()
    c.close()


@pytest.mark.parametrize("first,count,Hkv,G", SHAPES)
def test_first_keys_that_count_for_nothing(first, count, Hkv, G):
    """Logits of minus infinity at the first 100 keys: rows that see others have these, the rest is 0 / 0."""
    c = Call(first, count, Hkv, G, seed=6)
    c.q[..., 3] = 1
    per_key(c, c.k_off, lambda at, rows: torch.where((torch.arange(D, device=DEV) == 3)[None] & (at < 100)[:, None], -math.inf, rows.double()).to(torch.bfloat16))
    c.run()
    torch.cuda.synchronize()
    o, lse, pv, p2 = c.want()
    at = torch.cat([torch.arange(f, f + n, device=DEV) for f, n in zip(first, count)])
    sees = at >= 100
    assert torch.isnan(c.out[:c.T][~sees].float()).all() and (c.lse[:c.T][~sees] == -math.inf).all()
    if sees.any():
        P.check_attention(c.out[:c.T][sees], c.lse[:c.T][sees], tuple(x[sees] for x in (o, lse, pv, p2)), "")
    c.close()


@pytest.mark.parametrize("first,count,Hkv,G", SHAPES)
def test_the_largest_values(first, count, Hkv, G):
    """V of up to 2^90, and logits that rise by 60 binary orders at key 200."""
    c = Call(first, count, Hkv, G, seed=7)
    c.q[..., 3] = 1
    per_key(c, c.v_off, lambda at, rows: (rows.double().clamp(-1, 1) * 2.0 ** 90).to(torch.bfloat16))
    per_key(c, c.k_off, lambda at, rows: torch.where((torch.arange(D, device=DEV) == 3)[None] & (at >= 200)[:, None], 472.0, rows.double()).to(torch.bfloat16))
    c.run()
    c.check()
    c.close()


@pytest.mark.parametrize("big", [-2.0 ** 60, 2.0 ** 60])
def test_logits_far_from_zero(big):
    """A single key far below (above) everything: the running maximum starts there."""
    c = Call([0], [200], 1, 4)
    c.q.fill_(2.0 ** 40)
    K = c.kv[c.k_off[0]:c.k_off[0] + 200 * D].view(200, D)
    K.zero_()
    K[0, 0] = big
    c.run()
    torch.cuda.synchronize()
    o, l, _, _ = c.want()
    assert torch.isfinite(o).all()
    assert torch.allclose(c.lse[:200].double(), l, rtol=1e-6, atol=1e-4)
    V = c.kv[c.v_off[0]:c.v_off[0] + 200 * D].view(200, D).double()
    assert ((c.out[:200].double() - o).abs() <= 2.0 ** -7 * V.abs().max()).all()
    c.close()


@pytest.mark.parametrize("first,count,G", [(0, 200, 4), (0, 200, 1), (70, 90, 8), (4000, 6, 4)])
@pytest.mark.parametrize("what", [math.inf, math.nan])
def test_what_is_not_finite_stays_with_the_rows_that_see_it(first, count, G, what):
    """V and K at the middle token of the chunk: earlier tokens' results are what they are without it, to the bit; later ones' as in 64 bits."""
    c = Call([first], [count], 1, G)
    c.run()
    torch.cuda.synchronize()
    before, lse = c.out.clone(), c.lse.clone()
    at = count // 2
    c.kv[c.v_off[0] + (first + at) * D + 5] = what
    c.kv[c.v_off[0] + (first + at) * D + 64] = -what
    c.run()
    torch.cuda.synchronize()
    assert torch.equal(c.out[:at], before[:at]) and torch.equal(c.lse, lse)
    odd = c.out[at:c.T, :, [5, 64]].float()
    assert torch.isnan(odd).all() if math.isnan(what) else ((odd[..., 0] == math.inf) & (odd[..., 1] == -math.inf)).all()
    rest = [d for d in range(D) if d not in (5, 64)]
    assert torch.equal(c.out[at:c.T][..., rest], before[at:c.T][..., rest])
    c.kv[c.v_off[0] + (first + at) * D + 5] = 0.0
    c.kv[c.v_off[0] + (first + at) * D + 64] = 0.0
    c.kv[c.k_off[0] + (first + at) * D + 7] = math.nan
    c.run()
    torch.cuda.synchronize()
    assert torch.equal(c.out[:at], before[:at]) and torch.isnan(c.out[at:c.T].float()).all() and torch.isnan(c.lse[at:c.T]).all()
    c.close()


def test_rows_behind_the_last_are_not_read():
    """NaN in the rows of a sequence's blocks that the call's tokens do not reach."""
    c = Call([0, 0], [300, 300], 2, 4)
    c.first, c.count = [10, 0], [91, 66]
    c.T = 157
    for b, n in ((0, 101), (1, 66)):
        for h in range(2):
            for off in (c.k_off, c.v_off):
                c.kv[off[b * 2 + h] + n * D:off[b * 2 + h] + 300 * D] = math.nan
    c.q = c.q[:157].contiguous()
    c.out, c.lse = c.out[:158].clone(), c.lse[:158].clone()
    c.run()
    c.check()
    c.close()


def test_a_row_of_infinitely_negative_logits():
    """As the formula: nothing but minus infinities to choose from gives NaN, and -inf for lse."""
    c = Call([0], [70], 1, 1)
    c.kv[c.k_off[0]:c.k_off[0] + 70 * D] = -math.inf
    c.q.fill_(1.0)
    c.run()
    torch.cuda.synchronize()
    assert torch.isnan(c.out[:70].float()).all() and (c.lse[:70] == -math.inf).all()
    c.close()


def test_offsets_past_32_bits():
    c = Call([2000], [50], 1, 4)
    room = 2050 * D
    big = torch.empty((2 ** 32 + 2 * room + 64,), dtype=torch.bfloat16, device=DEV)
    for off, to in ((c.k_off, 2 ** 32 + 8), (c.v_off, 2 ** 32 + room + 16)):
        big[to:to + room] = c.kv[off[0]:off[0] + room]
        off[0] = to
    c.kv = big
    c.run()
    c.check()
    c.close()


def test_the_longest_context():
    """2^24 positions: K and V blocks of 4 GiB, their last rows at offsets around 2^32."""
    n = 2 ** 24
    c = Call([n - 2], [2], 1, 1)
    c.run()
    torch.cuda.synchronize()
    s = torch.empty((2, n), dtype=torch.float64, device=DEV)
    K, V = (c.kv[o[0]:o[0] + n * D].view(n, D) for o in (c.k_off, c.v_off))
    for i in range(0, n, 2 ** 20):
        s[:, i:i + 2 ** 20] = c.q[:, 0].double() @ K[i:i + 2 ** 20].double().t().contiguous() / math.sqrt(D)
    s[0, n - 1] = -math.inf
    lse = torch.logsumexp(s, -1)
    p = (s - lse[:, None]).exp()
    o = sum(p[:, i:i + 2 ** 20] @ V[i:i + 2 ** 20].double() for i in range(0, n, 2 ** 20))
    p2 = sum(p[:, i:i + 2 ** 20].square() @ V[i:i + 2 ** 20].double().square() for i in range(0, n, 2 ** 20)).sqrt()
    assert ((c.lse[:2, 0].double() - lse).abs() <= 1e-4 + 1e-6 * lse.abs()).all()
    # independent roundings of 2^24 weights (six standard deviations), and of the output; 32-bit sums over pieces of the keys: 2^-12 of that size
    assert ((c.out[:2, 0].double() - o).abs() <= 6 * 2.0 ** -8 * p2 + 2.0 ** -8 * o.abs() + 2.0 ** -12 * p2).all()
    c.close()


def test_streams_and_graphs():
    """On a stream of its own, and captured: replays beside eager work, on new inputs, are the eager results."""
    c = Call([100, 0, 5000], [70, 300, 2], 2, 4)
    c.run()
    c.check()
    want = c.out.clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    c.out.zero_()
    s.wait_stream(torch.cuda.current_stream())
    c.run(stream=s)
    s.synchronize()
    assert torch.equal(c.out[:c.T], want[:c.T])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run()
    for i in range(3):
        c.q.copy_(torch.randn_like(c.q.float()).to(torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        got, lse = c.out.clone(), c.lse.clone()
        c.out.zero_()
        c.run()
        torch.cuda.synchronize()
        assert torch.equal(got[:c.T], c.out[:c.T]) and torch.equal(lse, c.lse)
        assert not torch.equal(got[:c.T], want[:c.T])
    c.close()


def test_same_results_every_time():
    c = Call([300, 0, 41000], [1500, 900, 3], 4, 4)
    c.run()
    torch.cuda.synchronize()
    want, lse = c.out.clone(), c.lse.clone()
    for _ in range(5):
        c.work.fill_(255)
        c.run()
        torch.cuda.synchronize()
        assert torch.equal(c.out, want) and torch.equal(c.lse, lse)
    c.close()


def test_a_long_list_of_sequences_captured():
    """More sequences than a launch's arguments hold: what a replay needs of them is in the graph and the work buffer."""
    first, count = [700 * (i % 9) for i in range(90)], [1 + 40 * (i % 4) for i in range(90)]
    c = Call(first, count, 2, 4)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run()
    first, count = list(first), list(count)
    for i in range(3):
        c.q.copy_(torch.randn_like(c.q.float()).to(torch.bfloat16))
        c.work.fill_(255)
        graph.replay()
        c.check(i)
        got = c.out.clone()
        c.run()                                  # eager between the replays, in the same work buffer
        torch.cuda.synchronize()
        assert torch.equal(got, c.out)
    c.close()


def test_two_calls_at_once():
    """Of one context on two streams, a work buffer each; pieces in both."""
    a, b = Call([30000, 4], [3, 400], 4, 4, seed=1), Call([100, 25000], [900, 70], 4, 4, seed=2)
    hc.hc_destroy(b.ctx)
    b.ctx = a.ctx                                # a's room is the larger
    a.run(), b.run()
    torch.cuda.synchronize()
    want = a.out.clone(), b.out.clone()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        for c in (a, b):
            c.out.fill_(7)
            c.work.fill_(255)
        for s in streams:
            s.wait_stream(torch.cuda.current_stream())
        for _ in range(4):
            a.run(stream=streams[0])
            b.run(stream=streams[1])
        torch.cuda.synchronize()
        assert torch.equal(a.out, want[0]) and torch.equal(b.out, want[1])
    a.check("a")
    b.check("b")
    a.close()
