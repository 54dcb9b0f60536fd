"""hc_prefill_attn where a piece of the keys, or a wave's half of them, begins with nothing but logits of minus infinity.  Run with `-m gpu` on an MI355X."""
import math

import pytest
import torch

import prompt_util as P
from test_gpu_prompt_attn import DEV, SHAPES, Call

pytestmark = pytest.mark.gpu
# element 3 of K, the only one of q that is not zero: logits of 132.6, 49.9 and 44.9 binary orders below zero
LOWEST, LOW, HIGH = -1040.0, -392.0, -352.0


def later_pieces(at, first, count):
    """Tiles of 64 keys: in the earlier half of the keys they begin with the lowest and go on with the high ones, which together outweigh the rest; in the
    later half they begin with minus infinities and go on with the low ones."""
    early, begin = at < (first + count) // 128 * 64, at % 64 < 32
    return torch.where(early, torch.where(begin, LOWEST, HIGH), torch.where(begin, -math.inf, LOW))


def earlier_pieces(at, first, count):
    """The other way round."""
    late, begin = at >= (first + count) // 128 * 64, at % 64 < 32
    return torch.where(late, torch.where(begin, LOWEST, HIGH), torch.where(begin, -math.inf, LOW))


def halves(at, first, count):
    """The first tile: minus infinities, then the lowest; the others: low ones, then high ones."""
    begin = at % 64 < 32
    return torch.where(at < 64, torch.where(begin, -math.inf, LOWEST), torch.where(begin, LOW, HIGH))


@pytest.mark.parametrize("first,count,Hkv,G", SHAPES + [([0], [1024], 8, 4), ([30000], [1], 1, 8), ([4000, 9000], [3, 40], 2, 2)])
@pytest.mark.parametrize("pattern", [later_pieces, earlier_pieces, halves])
def test_parts_of_the_keys_that_begin_with_minus_infinity(first, count, Hkv, G, pattern):
    """What a part weighs against another one must not hang on where its reference started."""
    c = Call(first, count, Hkv, G, seed=8)
    c.q.zero_()
    c.q[..., 3] = 1
    for b, (f, n) in enumerate(zip(first, count)):
        for h in range(Hkv):
            rows = c.kv[c.k_off[b * Hkv + h]:][:(f + n) * P.D].view(f + n, P.D)
            rows[:, 3] = pattern(torch.arange(f + n, device=DEV), f, n).to(torch.bfloat16)
    c.run()
    torch.cuda.synchronize()
    o, lse, pv, p2 = c.want()
    sees = torch.isfinite(lse[:, 0])
    assert torch.isnan(c.out[:c.T][~sees].float()).all() and (c.lse[:c.T][~sees] == -math.inf).all()
    if sees.any():
        P.check_attention(c.out[:c.T][sees], c.lse[:c.T][sees], tuple(x[sees] for x in (o, lse, pv, p2)), pattern.__name__)
    c.close()
