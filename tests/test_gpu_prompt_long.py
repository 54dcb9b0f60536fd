"""hc_prefill_attn over many keys, held to a bound that a wrong tile of V does not keep.  Run with `-m gpu` on an MI355X."""
import pytest
import torch

from prompt_long_util import check_long
from test_gpu_prompt_attn import Call

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("first,count,Hkv,G", [
    ([60001], [9], 8, 4), ([20011, 47777], [1, 8], 8, 4), ([90001], [3], 2, 8), ([30000], [700], 2, 1), ([131071], [1], 1, 1), ([8192], [512], 8, 4),
    ([12345, 0, 40000], [1, 3000, 17], 4, 2)])
def test_many_keys(first, count, Hkv, G):
    c = Call(first, count, Hkv, G, seed=sum(count))
    c.run()
    torch.cuda.synchronize()
    want = c.want()
    behind = torch.cat([torch.arange(f, f + n) for f, n in zip(first, count)]) >= 1000          # rows of fewer keys: see test_gpu_prompt_attn.py
    behind = behind.to(want[0].device)
    check_long(c.out[:c.T][behind], tuple(x[behind] for x in want), (first, count, Hkv, G))
    c.close()
