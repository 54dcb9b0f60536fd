"""What the sharp checks of the 4-bit cache's attention let through and what they do not, on outputs made here.  No GPU needed."""
import math

import pytest
import torch

import kvq_sharp_util as S

D = 128


def rows(n, G, seed):
    g = torch.Generator().manual_seed(seed)
    K = torch.randn((n, D), generator=g).to(torch.bfloat16).double()
    return torch.randn((G, D), generator=g).to(torch.bfloat16), K, torch.randn((n, D), generator=g).to(torch.bfloat16).double()


def cut(x):
    """x rounded towards zero to bf16."""
    return (x.float().view(torch.int32) & -65536).view(torch.float32).double()


def outputs(q, K, V, parts=3, leave=None):
    """out, lse and weights in 64 bits, the weights beside the first query head's largest logit in so many parts; without the rows `leave`."""
    s = q.double() @ K.t() / math.sqrt(D)
    top = s[:, :1]                                               # (a reference that is not the largest: weights with all of their bits)
    w = torch.exp(s - top).float().double()
    held, rest = torch.zeros_like(w), w
    for _ in range(parts):
        held, rest = held + cut(rest), rest - cut(rest)
    if leave is not None:
        held[:, leave] = 0
    total = held.sum(-1)
    return (held @ V / total[:, None]).float(), (top[:, 0] + total.log()).float(), (w / w.sum(-1, keepdim=True)).mean(0).float()


@pytest.mark.parametrize("G", [1, 8])
@pytest.mark.parametrize("n", [100, 3000, 60000])
def test_rms(G, n):
    q, K, V = rows(n, G, n)
    S.check_rms(*outputs(q, K, V), q, K, V, "")
    for kw in (dict(parts=2), dict(leave=slice(32, 64)), dict(leave=slice(n - 1, n))):
        out, lse, w = outputs(q, K, V, **kw)
        with pytest.raises(AssertionError):
            S.check_rms(out, lse, w, q, K, V, "")
        with pytest.raises(AssertionError):                      # by the outputs alone
            S.check_rms(out, torch.logsumexp(q.double() @ K.t() / math.sqrt(D), -1).float(), w, q, K, V, "")
    out, lse, w = outputs(q, K, V)
    with pytest.raises(AssertionError):
        S.check_rms(out, lse, w * (1 + 2.0 ** -16 * torch.rand(n, generator=torch.Generator().manual_seed(1))), q, K, V, "")


@pytest.mark.parametrize("run", S.RUNS)
@pytest.mark.parametrize("n", [1, 31, 1000, 5000, 300000])
def test_ones(n, run):
    count = torch.bincount(S.column(n, run), minlength=D).double()

    def call(count, total=n, weights=n):
        S.check_ones((count / total).float()[None], torch.tensor([math.log(total)]).float(), torch.full((n,), 1 / weights), n, run, "")
    call(count)
    for lost in {1, min(32, n)}:
        for at in (0, n - lost):
            less = count - torch.bincount(S.column(n, run)[at:at + lost], minlength=D)
            if n > lost:
                with pytest.raises(AssertionError):
                    call(less, n - lost)
            with pytest.raises(AssertionError):
                call(less)
            if n > 2 * 4096:                                     # one twice in another's place
                twice = less + torch.bincount(S.column(n, run)[4096:4096 + lost], minlength=D)
                if not torch.equal(twice, count):
                    with pytest.raises(AssertionError):
                        call(twice)
    if n > 1:
        with pytest.raises(AssertionError):
            call(count, weights=n - 1)
