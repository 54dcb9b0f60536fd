"""hc_prefill_attn where logits are so large that their rounding to 32 bits passes whole binary orders.  Run with `-m gpu` on an MI355X."""
import math

import pytest
import torch

import prompt_util as P
from test_gpu_prompt_attn import DEV, SHAPES, Call

pytestmark = pytest.mark.gpu


def mantissas(n, seed):
    """n factors in [1, 2) of eight bits, few of them a power of two."""
    g = torch.Generator().manual_seed(seed)
    return 1 + torch.randint(0, 128, (n,), generator=g).to(DEV).double() / 128


def want(c):
    """As prompt_util.attention, the weights divided by their sum: from 2^52 on a row's lse in 64 bits is its largest logit, and exp(s - lse) adds up to the
    number of keys that have it."""
    T, H = c.T, c.Hkv * c.G
    o, pv, p2 = (torch.zeros((T, H, P.D), dtype=torch.float64, device=DEV) for _ in range(3))
    lse = torch.zeros((T, H), dtype=torch.float64, device=DEV)
    t = 0
    for b, (f, n) in enumerate(zip(c.first, c.count)):
        hidden = (torch.arange(f + n, device=DEV)[None] > torch.arange(f, f + n, device=DEV)[:, None])
        for a in range(H):
            K, V = (c.kv[off[b * c.Hkv + a // c.G]:][:(f + n) * P.D].view(f + n, P.D).double() for off in (c.k_off, c.v_off))
            s = (c.q[t:t + n, a].double() @ K.t().contiguous() / math.sqrt(P.D)).masked_fill(hidden, -math.inf)
            p = torch.softmax(s, -1)
            o[t:t + n, a], pv[t:t + n, a], p2[t:t + n, a], lse[t:t + n, a] = p @ V, p @ V.abs(), (p.square() @ V.square()).sqrt(), torch.logsumexp(s, -1)
        t += n
    return o, lse, pv, p2


@pytest.mark.parametrize("first,count,Hkv,G", SHAPES)
@pytest.mark.parametrize("e", [20, 22, 23, 24, 26, 28, 30, 31, 32, 33, 34, 40, 60, 100, 124])
def test_a_few_keys_far_above_the_rest(first, count, Hkv, G, e):
    """One element of q and K is not zero, so that a logit is one product of two bf16 numbers, exact in 32 bits: every 37th key above all others by 2^e
    or so, every fifth (to heads with negative queries: above) below them, the rest at zero.  Rows weigh the keys of the largest logit they see equally."""
    c = Call(first, count, Hkv, G, seed=e)
    q = mantissas(c.T * Hkv * G, e).view(c.T, Hkv, G) * 2.0 ** (e // 2)
    q[:, :, 1::2] *= -1
    c.q.zero_()
    c.q.view(c.T, Hkv, G, P.D)[..., 9] = q.to(torch.bfloat16)
    size = mantissas(2 * Hkv, e + 1) * 2.0 ** (e - e // 2)
    for b, (f, n) in enumerate(zip(first, count)):
        at = torch.arange(f + n, device=DEV)
        for h in range(Hkv):
            rows = c.kv[c.k_off[b * Hkv + h]:][:(f + n) * P.D].view(f + n, P.D)
            rows.zero_()
            rows[:, 9] = torch.where(at % 37 == 5, size[2 * h], torch.where(at % 5 == 0, -size[2 * h + 1], 0.0)).to(torch.bfloat16)
    c.run()
    torch.cuda.synchronize()
    # lse: scale, product, reference and the factor back are rounded to 32 bits, 2^-21.9 in all: 1e-6 of it, as everywhere
    P.check_attention(c.out[:c.T], c.lse[:c.T], want(c), (first, count, e))
    c.close()


@pytest.mark.parametrize("k", [-1.37, 1.37])
@pytest.mark.parametrize("e", [60, 80])
def test_one_key_far_from_zero(k, e):
    """A single key far below (above) everything, in the row that sees nothing else too."""
    c = Call([0], [200], 1, 4)
    c.q.fill_(1.1 * 2.0 ** 40)
    K = c.kv[c.k_off[0]:c.k_off[0] + 200 * P.D].view(200, P.D)
    K.zero_()
    K[0, 0] = k * 2.0 ** e
    c.run()
    torch.cuda.synchronize()
    P.check_attention(c.out[:200], c.lse[:200], want(c), (k, e))
    c.close()


@pytest.mark.parametrize("first,count,Hkv,G", SHAPES)
@pytest.mark.parametrize("e", [20, 24, 26, 28, 30, 31, 32, 33, 34, 36, 40, 60, 100, 124])
@pytest.mark.parametrize("sign", [1, -1])
def test_neighbouring_logits(first, count, Hkv, G, e, sign):
    """Logits one step of 32 bits apart (two products, their sum exact): by e the step is nothing, a few binary orders, or all the difference there is.  Half of the
    heads have their logits just below a power of two, where a step of the logit is less than one of the logit in binary orders."""
    c = Call(first, count, Hkv, G, seed=e)
    c.q.zero_()
    q = c.q.view(c.T, Hkv, G, P.D)
    q[..., 9], q[..., 10] = sign * 2.0 ** (e // 2), 2.0 ** (e // 2 - 20)
    for b, (f, n) in enumerate(zip(first, count)):
        step = (torch.arange(f + n, device=DEV) * 7 % 11 - 5).to(torch.bfloat16)
        for h in range(Hkv):
            rows = c.kv[c.k_off[b * Hkv + h]:][:(f + n) * P.D].view(f + n, P.D)
            rows.zero_()
            rows[:, 9] = (1.984375 if h % 2 == 0 else 1.40625) * 2.0 ** (e - e // 2)
            rows[:, 10] = step * 2.0 ** (e - e // 2 - 3)
    c.run()
    torch.cuda.synchronize()
    P.check_attention(c.out[:c.T], c.lse[:c.T], want(c), (first, count, e))
    c.close()
