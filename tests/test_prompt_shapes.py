"""What the binding of the operators in front of the cache refuses because it is not of the context's shape.  No GPU needed: the library's calls are stand-ins."""
import types

import pytest
import torch

from paper_2601_13684_amd import binding as hc

CTX, B, Hq, Hkv, D = 77, 3, 8, 2, 128


@pytest.fixture
def calls(monkeypatch):
    """The names of the calls that get as far as the library."""
    made = []

    def create(cfg, out):
        out._obj.value = CTX
        return hc.HC_OK
    fake = {n: (lambda n: lambda *a: made.append(n) or hc.HC_OK)(n) for n in ("hc_prefill_rope", "hc_prefill_attn", "hc_append_rope", "hc_destroy")}
    monkeypatch.setattr(hc, "lib", lambda: types.SimpleNamespace(hc_create=create, **fake))
    monkeypatch.setattr(hc, "_stream", lambda s: 0)
    assert hc.hc_create(hc.hc_config(B=B, Hq=Hq, Hkv=Hkv, D=D, max_ctx=64)) == CTX
    yield made
    hc.hc_destroy(CTX)


def heads(tokens, n):
    return torch.zeros((tokens, n, D), dtype=torch.bfloat16)


def rope(first=(0, 0, 0), count=(2, 0, 3), q=Hq, k=Hkv, v=Hkv, q_out=None, offsets=None):
    T = sum(count)
    off = [8 * i for i in range(len(first) * k if offsets is None else offsets)]
    hc.hc_prefill_rope(CTX, hc.hc_rope(), heads(T, q), heads(T, k), heads(T, v), first, count, heads(T, q) if q_out is None else q_out, 4096, off, off)


def attn(first=(0, 0, 0), count=(2, 0, 3), q=5 * Hq, out=5 * Hq, lse=5 * Hq, offsets=B * Hkv):
    off = [8 * i for i in range(offsets)]
    hc.hc_prefill_attn(CTX, heads(q, 1), 4096, off, off, first, count, heads(out, 1), None if lse is None else torch.zeros(lse), 4096, 1 << 40)


def append(tokens=B, q=Hq, k=Hkv, v=Hkv, q_out=B * Hq):
    hc.hc_append_rope(CTX, 1, hc.hc_rope(), heads(tokens, q), heads(tokens, k), heads(tokens, v), heads(q_out, 1), 4096)


@pytest.mark.parametrize("call,name", [(rope, "hc_prefill_rope"), (attn, "hc_prefill_attn"), (append, "hc_append_rope")])
def test_calls_of_the_right_shape(calls, call, name):
    call()
    assert calls == [name]


@pytest.mark.parametrize("kw", [dict(q=4), dict(q=16), dict(v=1), dict(v=4), dict(k=1), dict(k=4), dict(first=(0, 0), count=(2, 3)), dict(first=(0,) * 4, count=(2, 3, 0, 0)),
                                dict(q_out=heads(4, Hq)), dict(offsets=5)])
def test_refused_prompts(calls, kw):
    with pytest.raises(ValueError):
        rope(**kw)
    assert not calls


@pytest.mark.parametrize("kw", [dict(q=5 * Hq - 1), dict(out=5 * Hq - 1), dict(lse=5 * Hq - 1), dict(first=(0, 0), count=(2, 3), offsets=4), dict(offsets=3),
                                dict(first=(0,) * 4, count=(2, 3, 0, 0), offsets=8)])
def test_refused_attention(calls, kw):
    with pytest.raises(ValueError):
        attn(**kw)
    assert not calls


@pytest.mark.parametrize("kw", [dict(tokens=1, q_out=B * Hq), dict(tokens=2), dict(tokens=4, q_out=4 * Hq), dict(q=4), dict(q=9, q_out=27), dict(k=1), dict(v=1), dict(v=3), dict(q_out=B * Hq - 1)])
def test_refused_appends(calls, kw):
    """One row for three sequences among them: it was read as the row of every one."""
    with pytest.raises(ValueError):
        append(**kw)
    assert not calls


def test_one_row_for_every_sequence_is_said_by_a_stride_of_zero(calls):
    q, k, v = (heads(1, n).expand(B, -1, -1) for n in (Hq, Hkv, Hkv))
    hc.hc_append_rope(CTX, 1, hc.hc_rope(), q, k, v, 4096, 4096)
    hc.hc_prefill_attn(CTX, 4096, 4096, [0] * 6, [0] * 6, [0] * 3, [1] * 3, 1 << 20, None, 4096, 1 << 40)          # bare addresses are the caller's
    assert calls == ["hc_append_rope", "hc_prefill_attn"]


def test_larger_tensors_than_the_call_needs(calls):
    attn(q=6 * Hq, out=6 * Hq, lse=6 * Hq)
    attn(lse=None)
    rope(q_out=heads(6, Hq))
    append(q_out=B * Hq + 1)
    assert len(calls) == 4


def test_outputs_over_the_queries(calls):
    """Parts of the keys are read against q until the last of them is through."""
    x, off = heads(9, Hq), [8 * i for i in range(B * Hkv)]
    for q, out in ((x[:5], x[:5]), (x[:5], x[4:]), (x[4:], x[:5]), (x.data_ptr(), x)):
        with pytest.raises(ValueError, match="overlaps"):
            hc.hc_prefill_attn(CTX, q, 4096, off, off, [0] * 3, [2, 0, 3], out, None, 4096, 1 << 40)
    assert not calls
    hc.hc_prefill_attn(CTX, x[:5], 4096, off, off, [0] * 3, [1, 0, 3], x[4:], None, 4096, 1 << 40)
    hc.hc_prefill_attn(CTX, x, 4096, off, off, [0] * 3, [0] * 3, x, None, 4096, 1 << 40)             # nothing is read or written
    assert len(calls) == 2
