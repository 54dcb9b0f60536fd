"""What the binding of the 4-bit cache refuses because it is not of its table's shape or type.  No GPU needed: the library's calls are stand-ins."""
import types
from array import array

import pytest
import torch

from paper_2601_13684_amd import binding as hc

CTX, KVQ, TO, B, Hq, Hkv, D = 77, 1001, 1002, 3, 8, 2, 128


@pytest.fixture
def calls(monkeypatch):
    """The names of the calls that get as far as the library."""
    made, handles = [], [TO, KVQ]

    def create(cfg, out):
        out._obj.value = CTX
        return hc.HC_OK

    def table(ctx, heads, out):
        out._obj.value = handles.pop()
        return hc.HC_OK
    names = ("hc_kvq_store", "hc_kvq_load", "hc_kvq_append", "hc_kvq_attn", "hc_kvq_evict", "hc_kvq_destroy", "hc_destroy")
    fake = {n: (lambda n: lambda *a: made.append(n) or hc.HC_OK)(n) for n in names}
    monkeypatch.setattr(hc, "lib", lambda: types.SimpleNamespace(hc_create=create, hc_kvq_create=table, **fake))
    monkeypatch.setattr(hc, "_stream", lambda s: 0)
    assert hc.hc_create(hc.hc_config(B=B, Hq=Hq, Hkv=Hkv, D=D, max_ctx=64)) == CTX
    assert hc.hc_kvq_create(CTX, heads(64)) == KVQ and hc.hc_kvq_create(CTX, heads(16)) == TO
    yield made
    made.clear()
    hc.hc_kvq_destroy(KVQ)
    hc.hc_kvq_destroy(TO)
    hc.hc_destroy(CTX)
    assert KVQ not in hc._tables and TO not in hc._tables


def heads(cap, n=B * Hkv):
    return [hc.hc_kvq_head(off=136 * cap * i, row_off=cap * i, cap=cap, budget=cap) for i in range(n)]


def u8(n):
    return torch.zeros((n,), dtype=torch.uint8)


def state(n=B * Hkv, t=torch.int32):
    return torch.zeros((n, 2), dtype=t)


def f32(*n):
    return torch.zeros(n)


def bf16(*n):
    return torch.zeros(n, dtype=torch.bfloat16)


SIZE, ROWS, OFF = 136 * 64 * B * Hkv, 64 * B * Hkv, [8 * i for i in range(B * Hkv)]


def store(first=(0, 0, 0), count=(2, 0, 3), off=OFF, arena=SIZE, st=None, acc=ROWS):
    hc.hc_kvq_store(CTX, KVQ, 4096, off, off, first, count, u8(arena), state() if st is None else st, None if acc is None else f32(acc))


def load(first=(0, 0, 0), count=(2, 0, 3), off=OFF, arena=SIZE, st=None):
    hc.hc_kvq_load(CTX, KVQ, u8(arena), state() if st is None else st, first, count, 4096, off, off)


def append(tokens=B, q=Hq, k=Hkv, v=Hkv, out=None, arena=SIZE, st=None, acc=ROWS):
    hc.hc_kvq_append(CTX, KVQ, hc.hc_rope(), bf16(tokens, q, D), bf16(tokens, k, D), bf16(tokens, v, D), bf16(B, Hq, D) if out is None else out, u8(arena),
                     state() if st is None else st, f32(acc))


def attn(arena=SIZE, st=None, q=None, out=None, lse=None, acc=ROWS, work=64, said=64):
    hc.hc_kvq_attn(CTX, KVQ, u8(arena), state() if st is None else st, bf16(B, Hq, D) if q is None else q, f32(B, Hq, D) if out is None else out,
                   f32(B, Hq) if lse is None else lse, None if acc is None else f32(acc), 1.0, u8(work), said)


def evict(arena=SIZE, acc=ROWS, to_arena=SIZE // 4, to_st=None, to_acc=ROWS // 4, kept=None):
    hc.hc_kvq_evict(CTX, KVQ, u8(arena), state(), f32(acc), TO, u8(to_arena), state() if to_st is None else to_st, f32(to_acc), kept, u8(64), 64)


@pytest.mark.parametrize("call", [store, load, append, attn, evict])
def test_calls_of_the_right_shape(calls, call):
    call()
    assert calls == ["hc_kvq_" + call.__name__]


@pytest.mark.parametrize("call,kw", [
    (store, dict(first=(0, 0))), (store, dict(first=(0, 0), count=(1, 1))), (store, dict(off=OFF[:-1])), (store, dict(off=OFF[:3])), (store, dict(arena=SIZE - 1)),
    (store, dict(st=state(5))), (store, dict(st=state(t=torch.int64))), (store, dict(acc=ROWS - 1)),
    (load, dict(count=(1, 1))), (load, dict(off=OFF * 2)), (load, dict(arena=SIZE - 1)), (load, dict(st=state(5))),
    (append, dict(tokens=2)), (append, dict(q=4)), (append, dict(k=1)), (append, dict(v=3)), (append, dict(out=bf16(B, Hq - 1, D))), (append, dict(out=f32(B, Hq, D))),
    (append, dict(arena=SIZE - 1)), (append, dict(st=state(5))), (append, dict(acc=ROWS - 1)),
    (attn, dict(arena=SIZE - 1)), (attn, dict(st=state(5))), (attn, dict(q=f32(B, Hq, D))), (attn, dict(q=bf16(B, 1, D))), (attn, dict(out=bf16(B, Hq, D))),
    (attn, dict(out=f32(B, Hq, 64))), (attn, dict(lse=f32(B))), (attn, dict(acc=ROWS - 1)), (attn, dict(work=63)),
    (evict, dict(arena=SIZE - 1)), (evict, dict(acc=ROWS - 1)), (evict, dict(to_arena=SIZE // 4 - 1)), (evict, dict(to_st=state(5))), (evict, dict(to_acc=ROWS // 4 - 1)),
    (evict, dict(kept=torch.zeros((ROWS // 4 - 1,), dtype=torch.int32))), (evict, dict(kept=torch.zeros((ROWS,), dtype=torch.int64)))])
def test_refused(calls, call, kw):
    with pytest.raises(ValueError):
        call(**kw)
    assert not calls


def test_nothing_accumulated_and_no_list(calls):
    store(acc=None)
    attn(acc=None)
    evict(kept=torch.zeros((ROWS // 4,), dtype=torch.int32))
    assert len(calls) == 3


def test_a_table_of_other_heads(calls):
    with pytest.raises(ValueError):
        hc.hc_kvq_create(CTX, heads(16, 5))


def test_long_lists():
    x = [i * 2 ** 30 for i in range(512)]
    assert hc._ints(x, "q") == array("q", x) and hc._ints(list(range(100)), "i") == array("i", range(100))
    with pytest.raises(OverflowError):
        hc._ints([0] * 40 + [2 ** 31], "i")
    with pytest.raises(TypeError):
        hc._ints([0] * 40 + [1.5], "q")
