"""Streams of the cache held in 4 bits where its work buffer is another cache's, or the program's own: what a call on some stream waits for, and what is kept until it
is through.  No GPU needed (torch's streams and the calls of the library are stand-ins that write down what they are asked for)."""
import types

import pytest

import test_prompt_streams as S
from paper_2601_13684_amd import runtime as R
from test_prompt_streams import Stream, log, on

CALLS = ("hc_kvq_attn", "hc_kvq_evict", "hc_kvq_append", "hc_kvq_store", "hc_kvq_load")


@pytest.fixture
def table(monkeypatch):
    log.clear()
    del S.now[1:], S.capturing[:]
    cuda = types.SimpleNamespace(Stream=Stream, Event=S.Event, ExternalStream=Stream, stream=on, current_stream=lambda device=None: S.now[-1],
                                 is_current_stream_capturing=lambda: S.now[-1].cuda_stream in S.capturing)
    make = lambda kind: lambda shape, **kw: S.Tensor(kind, shape, **kw)  # noqa: E731
    monkeypatch.setattr(R, "torch", types.SimpleNamespace(cuda=cuda, empty=make("empty"), zeros=make("zeros"), bfloat16=0, float32=0, uint8=0, int32=0, Tensor=S.Tensor))
    monkeypatch.setattr(R, "hc", types.SimpleNamespace(hc_rope=None, **{n: (lambda n: lambda *a: log.append((n, a[-1])))(n) for n in CALLS}))
    ctx = types.SimpleNamespace(handle=1, device="cuda:0", cfg=types.SimpleNamespace(B=1, Hq=4, Hkv=1))
    return types.SimpleNamespace(ctx=ctx, handle=2, nbytes=136 * 16, rows=16, heads=[None], work_bytes=lambda: 4096)


def attn(cache, stream):
    cache.attn(object(), stream=stream)


def evict(cache, stream):
    cache.evict(R.QuantCache(cache.table), stream=stream)


def asked(call, cache, stream):
    """(events waited for, by what was queued before them; what was kept) on the stream, in front of the call."""
    start = len(log)
    call(cache, stream)
    at = next(i for i in range(start, len(log)) if log[i][0].startswith("hc_kvq"))
    handle = stream.cuda_stream
    return [e[2] for e in log[start:at] if e[:2] == ("wait", handle)], [e[2] for e in log[start:at] if e[:2] == ("keep", handle)]


@pytest.mark.parametrize("call", [attn, evict])
@pytest.mark.parametrize("made_there", [False, True])
def test_another_caches_work_buffer(table, call, made_there):
    """The owner is made on the default stream; the cache that uses its buffer on stream 7 is made there too, or on the default one."""
    owner = R.QuantCache(table)
    made = len(log)
    side = Stream(7)
    if made_there:
        with on(side):
            cache = R.QuantCache(table, work=owner.work)
    else:
        cache = R.QuantCache(table, work=owner.work)
    waits, kept = asked(call, cache, side)
    assert any(w >= made for w in waits)                         # the owner's buffers, and the last use of their memory, are in front of it
    assert owner.work in kept and (cache.arena in kept) == (not made_there)


@pytest.mark.parametrize("call", [attn, evict])
def test_a_work_buffer_of_the_programs_own(table, call):
    """Nothing tells which stream it was made on: it is kept for every one that it is used on."""
    work = S.Tensor("empty", (4096,))
    cache = R.QuantCache(table, work=work)
    for stream in (Stream(0), Stream(7)):
        assert work in asked(call, cache, stream)[1]


def test_the_owners_stream(table):
    """On the stream that both were made on, nothing is asked for, and an owned buffer is kept as the others are."""
    owner = R.QuantCache(table)
    cache = R.QuantCache(table, work=owner.work)
    assert asked(attn, cache, Stream(0)) == ([], []) and asked(attn, owner, Stream(0)) == ([], [])
    assert owner.work in asked(attn, owner, Stream(7))[1]


def test_nothing_while_a_graph_is_captured(table):
    owner = R.QuantCache(table)
    caches = [R.QuantCache(table, work=owner.work), R.QuantCache(table, work=S.Tensor("empty", (4096,)))]
    S.capturing.append(7)
    for cache in caches:
        assert asked(attn, cache, Stream(7)) == ([], [])
