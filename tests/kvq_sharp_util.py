"""Checks of attention over the cache held in 4 bits that one row, one tile of 32 rows or one part of a weight does not get past."""
import math

import torch

D = 128
RMS = 1.5e-6
# How the rows of a head are told apart: a row has a 1 in one column, by its number, its tile of 32, or its run of 128 tiles, and zeros elsewhere.
RUNS = (1, 32, 4096)


def column(n, run, dev="cpu"):
    return torch.arange(n, device=dev) // run % D


def put_ones(cache, i, run):
    """Head i's rows: K of zeros, V with a 1 a row."""
    n = int(cache.state[i, 0])
    if n == 0:
        return
    (kc, ks), (vc, vs) = cache.blocks(i, 0), cache.blocks(i, 1)
    kc[:n], ks[:n], vc[:n], vs[:n] = 0, 127, 0, 127
    at = column(n, run, vc.device)
    vc[torch.arange(n, device=vc.device), at // 2] = (2 << 4 * (at % 2)).to(torch.uint8)         # (code 2 is 1)


def check_ones(out, lse, weights, n, run, where):
    """out [G, 128], lse [G] and the rows' weights [n] (or None) of a head of put_ones: every logit is 0, every weight 1 and every sum a whole number below 2^24, exact
    in 32 bits.  What is divided is off by a division's step or two, 2^-22 of itself; lse by a logarithm's and a product's, 2^-22 too."""
    want = torch.bincount(column(n, run, out.device), minlength=D).double() / n
    assert ((out.double() - want).abs() <= 2.0 ** -22 * want).all(), (where, n, run, float((out.double() - want).abs().max()))
    assert ((lse.double() - math.log(n)).abs() <= 2.0 ** -22 * math.log(n) + 1e-30).all(), (where, n, "lse")
    if weights is not None:
        assert ((weights.double() * n - 1).abs() <= 2.0 ** -22).all(), (where, n, "weights")


def check_rms(out, lse, weights, q, K, V, where):
    """out [G, 128], lse [G] and the rows' weights [n] (or None) of queries q [G, 128] over rows K, V, logits of a few units.  A logit up to 5 is off by roundings of its sums, each at
    most 2^-24 of it, some ten of them, as independent ones 6e-7 at the most; the difference's product, the factor and the exponential add 3e-7: a weight is off by less than 7e-7 of itself as a rule, an output
    by as much of its own size, since weights' errors and values have nothing to do with each other, and the sums over rows by a step or two of 32 bits.  Of a weight in two parts of
    bf16, 2^-15 of it at most is lost, 6e-6 as a rule; of n rows, a lost tile is 32 / n of an lse, one in sqrt(n / 32) of an output."""
    s = q.double() @ K.t().contiguous() / math.sqrt(D)
    p, l = torch.softmax(s, -1), torch.logsumexp(s, -1)
    want = p @ V
    rms = ((out.double() - want).square().mean(-1) / want.square().mean(-1)).sqrt()
    assert (rms <= RMS).all(), (where, len(K), rms)
    assert ((lse.double() - l).abs() <= 1e-6 + 2.0 ** -23 * l.abs()).all(), (where, len(K), "lse", lse.double() - l)
    if weights is not None:
        mean = p.mean(0)
        rms = float(((weights.double() / mean - 1).square().mean()).sqrt())
        assert rms <= RMS, (where, len(K), "weights", rms)
