"""What the bounds of the long-context tests let pass.  No GPU needed."""
import pytest
import torch

from prompt_long_util import attention, check_long

N, G, D = 20000, 4, 128


def case(seed=0):
    g = torch.Generator().manual_seed(seed)
    q = torch.randn((1, G, D), generator=g).to(torch.bfloat16)
    kv = torch.randn((2 * N * D,), generator=g).to(torch.bfloat16)
    return q, kv


def as_the_kernel(q, kv):
    """Weights rounded to bf16 for the second product, their sum from the unrounded ones, one rounding of the output."""
    k, v = kv.view(2, N, D).double()
    s = q[0].double() @ k.t() / D ** 0.5
    w = torch.exp(s - s.amax(-1, keepdim=True)).float()
    return (w.to(torch.bfloat16).double() @ v / w.double().sum(-1, keepdim=True)).to(torch.bfloat16)[None]


def test_right_outputs_pass():
    q, kv = case()
    check_long(as_the_kernel(q, kv), attention(q, kv, [0], [N * D], [N - 1], [1], 1, G), "")


@pytest.mark.parametrize("tile", [0, 100, 310])
@pytest.mark.parametrize("how", ["another tile's", "a row further", "nothing"])
def test_a_wrong_tile_of_values_does_not(tile, how):
    """The mistake is in what the outputs are compared with."""
    q, kv = case()
    out, wrong = as_the_kernel(q, kv), kv.clone()
    v, w = kv.view(2, N, D)[1], wrong.view(2, N, D)[1]
    at = slice(64 * tile, 64 * tile + 64)
    w[at] = {"another tile's": v[64 * tile + 64:64 * tile + 128], "a row further": v[64 * tile + 1:64 * tile + 65], "nothing": 0 * v[at]}[how]
    with pytest.raises(AssertionError):
        check_long(out, attention(q, wrong, [0], [N * D], [N - 1], [1], 1, G), "")
