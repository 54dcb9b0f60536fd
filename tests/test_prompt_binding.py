"""What the binding of the operators in front of the cache takes and refuses by itself.  No GPU needed."""
from array import array

import pytest
import torch

from paper_2601_13684_amd import binding as hc


def test_heads_of_views():
    x = torch.zeros((5, 12, 128), dtype=torch.bfloat16)
    q, k, v = x[:, :8], x[:, 8:10], x[:, 10:]
    assert hc._qkv(q, k, v) == (x.data_ptr(), x.data_ptr() + 8 * 256, x.data_ptr() + 10 * 256, 12 * 128, 12 * 128, 12 * 128, hc.HC_BF16)
    one = torch.zeros((1, 4, 128)).expand(5, -1, -1)
    assert hc._heads(one)[1] == 0
    assert hc._heads(torch.zeros((1, 12, 128))[:, :3])[1:] == (0, 1)           # a single token has no step
    assert hc._qkv(*(t.float() for t in (q, k, v)))[6] == hc.HC_F32


@pytest.mark.parametrize("bad", [
    lambda x: x[:, :, :64], lambda x: x[:, ::2], lambda x: x.transpose(0, 1), lambda x: x[:, :, 0], lambda x: x.view(5, 6, 256)])
def test_refused_heads(bad):
    with pytest.raises(ValueError):
        hc._heads(bad(torch.zeros((5, 12, 128))))


def test_refused_sets():
    x = torch.zeros((5, 4, 128))
    for q, k, v in ((x, x.half(), x), (x, x, x[:4]), (x.half(),) * 3, (x.double(),) * 3):
        with pytest.raises(ValueError):
            hc._qkv(q, k, v)
    for first, count, k_off, v_off in (([0], [1, 2], [0], [0]), ([0], [1], [0, 8], [0]), ([0, 0], [1, 1], [0, 8, 16], [0, 8, 16])):
        with pytest.raises(ValueError):
            hc._chunks(first, count, k_off, v_off)


def test_lists_and_kept_arrays():
    keep = array("q", [0, 8])
    first, count, k_off, v_off = hc._chunks((3,), [4], keep, [16, 2 ** 40])
    assert k_off is keep and list(v_off) == [16, 2 ** 40] and first.typecode == "i" and list(count) == [4]
    with pytest.raises(OverflowError):
        hc._chunks([2 ** 31], [0], keep, keep)


def test_rope_holds_its_weights():
    w = torch.ones(128)
    r = hc.hc_rope_init(hc.HC_ROPE_HALF, 128, 10000.0, q_norm=w, eps=1e-5, gain=0.5)
    assert r.q_norm == w.data_ptr() and r.k_norm is None and r.keep[0] is w and r.gain == 0.5 and r.eps == pytest.approx(1e-5)
    for bad in (torch.ones(64), torch.ones(128, dtype=torch.bfloat16)):
        with pytest.raises(ValueError):
            hc.hc_rope_init(hc.HC_ROPE_HALF, 128, 10000.0, k_norm=bad)
