"""Attention over the cache held in 4 bits where logits are so large that their rounding to 32 bits passes whole binary orders.  Run with `-m gpu` on an MI355X."""
import math

import pytest
import torch

import kvq_util as U
from paper_2601_13684_amd import binding as hc

pytestmark = pytest.mark.gpu
D = 128
ROWS = [[700, 33], [700, 33], [5000, 0, 1, 1500]]
CAPS = [[1024, 1008], [2704, 2048], [6000, 1040, 2048, 1504]]      # one launch; two, with few rows; two, a head's rows on several workgroups


def mantissas(n, seed):
    """n factors in [1, 2) of eight bits, few of them a power of two."""
    g = torch.Generator().manual_seed(seed)
    return 1 + torch.randint(0, 128, (n,), generator=g).to(U.DEV).double() / 128


def made(which, G, seed):
    rows, caps = ROWS[which], CAPS[which]
    ctx = U.context(1, len(rows), G, max(caps))
    cache = U.Cache(ctx, caps, rows=rows)
    for i, n in enumerate(rows):
        if n:
            cache.put(i, 0, 0, torch.zeros((n, D), dtype=torch.bfloat16, device=U.DEV))
            cache.put(i, 1, 0, U.rows_of(n, seed + i))
    cache.acc = torch.rand((cache.rows,), generator=torch.Generator(device=U.DEV).manual_seed(seed), device=U.DEV)
    return ctx, cache


def check(ctx, cache, q, G, where):
    """A logit is exact: one product, or two whose sum 32 bits hold.  What is left of a weight x binary orders below the largest: its difference from a reference, and
    that reference's from the largest one, are at most x + 16 orders in all (a weight is at most 2^8 of its reference), each rounded, multiplied and the factor
    rounded: (x + 16) ln 2 * 3 * 2^-24 < (x + 16) 2^-22; four exponentials of 2^-22; the same of the sum that divides it, where x is 0: below
    (x + 64) 2^-22.  Sums over n rows: (n / 8 + 64) 2^-24 (see check_attention).  Weights beyond 40 orders come to nothing in a sum."""
    heads = len(cache.caps)
    out, lse = torch.full((heads, G, D), 9.0, device=U.DEV), torch.full((heads, G), 9.0, device=U.DEV)
    work = cache.work()
    work.fill_(0xff)
    before = cache.acc.clone()
    hc.hc_kvq_attn(ctx, cache.kvq, cache.arena, cache.state, q, out, lse, cache.acc, 0.5, work, work.numel())
    acc, before, q, out, lse = cache.acc.cpu(), before.cpu(), q.cpu(), out.cpu(), lse.cpu()       # (a GPU's powers of two are not all exact)
    for i, n in enumerate(cache.state[:, 0].tolist()):
        if n == 0:
            assert (out[i] == 0).all() and (lse[i] == -math.inf).all()
            continue
        K, V = (U.decode(*(x[:n].cpu() for x in cache.blocks(i, v))) for v in (0, 1))
        s = q.view(heads, G, D)[i].double() @ K.t().contiguous()                 # exact in 64 bits, and in 32
        assert torch.equal(s.float().double(), s)
        top = s.amax(-1, keepdim=True)
        x = (s - top) / math.sqrt(D)
        p = torch.softmax(x, -1)
        l = torch.logsumexp(x, -1) + top[:, 0] / math.sqrt(D)
        sums = (n / 8 + 64) * 2.0 ** -24
        err = (out[i].double() - p @ V).abs()
        assert (err <= (104 * 2.0 ** -22 + sums) * (p @ V.abs()) + 1e-38).all(), (where, i, float(err.max()))
        assert ((lse[i].double() - l).abs() <= 64 * 2.0 ** -22 + sums + 2.0 ** -22 * l.abs()).all(), (where, i, lse[i], l)
        r = cache.heads[i].row_off
        rel = (64 - x / math.log(2)) * 2.0 ** -22 + sums
        want = before[r:r + n].double() * 0.5 + p.mean(0)
        err = (acc[r:r + n].double() - want).abs()
        assert (err <= (rel.clamp(max=1) * p).mean(0) + 2.0 ** -22 * want + 1e-37).all(), (where, i, float(err.max()))
    cache.close()
    hc.hc_destroy(ctx)


@pytest.mark.parametrize("which", [0, 1, 2])
@pytest.mark.parametrize("G", [1, 2, 4, 8])
@pytest.mark.parametrize("e", [10, 20, 24, 28, 30, 31, 32, 33, 34, 36, 40, 60, 100, 124, 126])
def test_a_few_rows_far_above_the_rest(which, G, e):
    """One element of q and K is not zero: every 37th row above all others by 2^e or so, every fifth (to queries of the other sign: above) below them, the rest at zero.  The
    rows of the largest logit weigh the same."""
    ctx, cache = made(which, G, e)
    heads = len(cache.caps)
    q = torch.zeros((heads * G, D), dtype=torch.float64, device=U.DEV)
    q[:, 9] = mantissas(heads * G, e) * 2.0 ** (e // 2)
    q[1::2] *= -1
    for i, n in enumerate(ROWS[which]):
        at = torch.arange(n, device=U.DEV)
        x = torch.zeros((n, D), dtype=torch.float64, device=U.DEV)
        x[:, 9] = torch.where(at % 37 == 5, 1.5 if i % 2 else 1.0, torch.where(at % 5 == 0, -1.0 if i % 2 else -1.5, 0.0)) * 2.0 ** (e - e // 2)
        cache.put(i, 0, 0, x.to(torch.bfloat16))
    check(ctx, cache, q.to(torch.bfloat16), G, (which, G, e))


@pytest.mark.parametrize("which", [0, 1, 2])
@pytest.mark.parametrize("G", [1, 4, 8])
@pytest.mark.parametrize("e", [20, 24, 26, 28, 30, 31, 32, 33, 34, 36, 40, 60, 100, 124])
@pytest.mark.parametrize("sign", [1, -1])
def test_neighbouring_logits(which, G, e, sign):
    """Logits of 2^e to 1.5 * 2^e, of either sign, that are equal or one step of 32 bits apart: by e the step is nothing, a few binary orders, or all the difference there is."""
    ctx, cache = made(which, G, e)
    heads = len(cache.caps)
    q = torch.zeros((heads * G, D), dtype=torch.float64, device=U.DEV)
    q[:, 9], q[:, 70] = sign * 2.0 ** (e // 2), 2.0 ** (e // 2 - 12)
    q[1::2, 9] *= 1.25
    for i, n in enumerate(ROWS[which]):
        at = torch.arange(n, device=U.DEV)
        x = torch.zeros((n, D), dtype=torch.float64, device=U.DEV)
        x[:, 9] = 2.0 ** (e - e // 2)
        x[:, 70] = torch.where((at * 7919) % 11 < 4, 2.0 ** (e - e // 2 - 11), 0.0)
        cache.put(i, 0, 0, x.to(torch.bfloat16))
    check(ctx, cache, q.to(torch.bfloat16), G, (which, G, e, sign))


@pytest.mark.parametrize("which", [0, 1, 2])
@pytest.mark.parametrize("G", [1, 4, 8])
@pytest.mark.parametrize("e", [31, 36, 60, 124])
def test_every_row_the_same_far_logit(which, G, e):
    """Every row weighs 1 / n, whichever side of zero the logits are on and whatever their rounded products would be off."""
    ctx, cache = made(which, G, e)
    heads = len(cache.caps)
    q = torch.zeros((heads * G, D), dtype=torch.float64, device=U.DEV)
    q[:, 9] = mantissas(heads * G, e + 3) * 2.0 ** (e // 2)
    q[::2] *= -1
    for i, n in enumerate(ROWS[which]):
        x = torch.zeros((n, D), dtype=torch.float64, device=U.DEV)
        x[:, 9] = 1.5 * 2.0 ** (e - e // 2)
        cache.put(i, 0, 0, x.to(torch.bfloat16))
    check(ctx, cache, q.to(torch.bfloat16), G, (which, G, e))
