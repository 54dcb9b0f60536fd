"""Streams of the prompt stage: what is queued, in which order, when a chunk or an initialisation is put on another stream than the one its buffers were made
on.  No GPU needed (torch's streams and the calls of the library are stand-ins that write down what they are asked for)."""
import contextlib
import types

import pytest

from paper_2601_13684_amd import runtime as R

log = []


class Stream:
    def __init__(self, handle, device=None):
        self.cuda_stream = int(handle)

    def wait_event(self, event):
        log.append(("wait", self.cuda_stream, event.after))


class Event:
    def record(self, stream):
        self.after = len(log)                    # what the log holds by now is in front of it


class Tensor:
    def __init__(self, kind, shape, device=None, dtype=None):
        self.shape = shape
        log.append((kind, now[-1].cuda_stream, self))

    def numel(self):
        return self.shape[0]

    def record_stream(self, stream):
        log.append(("keep", stream.cuda_stream, self))


now = [Stream(0)]
capturing = []


@contextlib.contextmanager
def on(stream):
    now.append(stream)
    yield
    now.pop()


@pytest.fixture
def prompt(monkeypatch):
    log.clear()
    del now[1:], capturing[:]
    cuda = types.SimpleNamespace(Stream=Stream, Event=Event, ExternalStream=Stream, stream=on, current_stream=lambda device=None: now[-1],
                                 is_current_stream_capturing=lambda: now[-1].cuda_stream in capturing)
    make = lambda kind: lambda shape, **kw: Tensor(kind, shape, **kw)  # noqa: E731
    monkeypatch.setattr(R, "torch", types.SimpleNamespace(cuda=cuda, empty=make("empty"), zeros=make("zeros"), bfloat16=0, float32=0, uint8=0))
    calls = types.SimpleNamespace(hc_prefill_attn_work_bytes=lambda ctx: 4096, hc_prefill_work_bytes=lambda ctx, layer: 64,
                                  **{n: (lambda n: lambda *a: log.append((n, a[-1])))(n) for n in ("hc_prefill_rope", "hc_prefill_attn")})
    monkeypatch.setattr(R, "hc", calls)
    ctx = types.SimpleNamespace(handle=1, device="cuda:0", cfg=types.SimpleNamespace(B=1, Hq=4, Hkv=1))
    return R.Prompt(ctx, [10])


def chunk(p, stream):
    made = len(log)
    x = types.SimpleNamespace(shape=(3, 4, 128))
    p.chunk(None, x, x, x, [3], stream)
    return log[:made], log[made:]


def names(entries):
    return [e[0] for e in entries]


@pytest.mark.parametrize("stream", [Stream(7), 7])
def test_a_chunk_on_another_stream(prompt, stream):
    before, after = chunk(prompt, stream)
    call = names(after).index("hc_prefill_rope")
    waits = [e for e in after[:call] if e[0] == "wait"]
    # it waits for everything that was queued with the buffers, and they are not given away before its work is through
    assert waits and waits[0][1] == 7 and waits[0][2] >= len([e for e in before if e[0] == "zeros"]) > 0
    assert {id(e[2]) for e in after[:call] if e[0] == "keep" and e[1] == 7} == {id(prompt.kv), id(prompt.work)}
    assert all(e[1] == 7 for e in after if e[0] == "empty")                    # the outputs are that stream's own


def test_a_chunk_under_another_current_stream(prompt):
    with on(Stream(9)):
        _, after = chunk(prompt, None)
    assert names(after).count("wait") == 1 and names(after).count("keep") == 2 and names(after).index("wait") < names(after).index("hc_prefill_rope")


@pytest.mark.parametrize("stream", [None, Stream(0), 0])
def test_a_chunk_on_the_same_stream(prompt, stream):
    _, after = chunk(prompt, stream)
    assert "wait" not in names(after) and "keep" not in names(after)


@pytest.mark.parametrize("given", [True, False])
def test_a_chunk_that_is_captured(prompt, given):
    """An event from outside of a capture cannot be waited for in it."""
    capturing.append(7)
    with contextlib.nullcontext() if given else on(Stream(7)):
        _, after = chunk(prompt, Stream(7) if given else None)
    assert "wait" not in names(after) and "keep" not in names(after)


def test_the_work_buffer_is_not_filled(prompt):
    assert [e[0] for e in log if e[2] is prompt.work] == ["empty"]


@pytest.mark.parametrize("stream", [Stream(7), 7])
def test_initialisation_on_another_stream(prompt, stream):
    lay = R.LayerRuntime.__new__(R.LayerRuntime)
    lay.ctx, lay.spec, lay.handle = prompt.ctx, types.SimpleNamespace(ctx=[0], B=1, Hkv=1), 2
    lay.arena = R.torch.zeros((5,))
    lay.topk_idx, lay.base_idx, lay.ring, lay.slot_pos = (R.torch.zeros((5,)) for _ in range(4))
    lay.made = R._Made("cuda:0")
    lay.prefill_init = lambda data, q, pool, stream: log.append(("init", stream, q))
    at = len(log)
    where = []
    lay.prefill_from(prompt, types.SimpleNamespace(to=lambda device: where.append(now[-1].cuda_stream) or "q"), 1, stream)
    after = log[at:]
    assert after[-1] == ("init", stream, "q") and where == [7]                 # a copy of the queries is that stream's
    assert [e[1] for e in after if e[0] == "wait"] == [7, 7] and max(e[2] for e in after if e[0] == "wait") == at
    assert {id(e[2]) for e in after if e[0] == "keep"} == {id(x) for x in (prompt.kv, lay.arena, lay.topk_idx, lay.base_idx, lay.ring, lay.slot_pos)}


@pytest.mark.parametrize("spec", [dict(ctx=[0], B=1, Hkv=2), dict(ctx=[1], B=1, Hkv=1), dict(ctx=[0, 0], B=2, Hkv=1)])
def test_a_prompt_of_another_shape(prompt, spec):
    """Its lists of offsets are as long as it has heads."""
    lay = R.LayerRuntime.__new__(R.LayerRuntime)
    lay.ctx, lay.spec = prompt.ctx, types.SimpleNamespace(**spec)
    lay.prefill_init = lambda *a: pytest.fail("taken")
    lay.made = R._Made("cuda:0")
    lay.handle = 2
    with pytest.raises(ValueError):
        lay.prefill_from(prompt, types.SimpleNamespace(to=lambda device: "q"))


def test_buffers_that_are_let_go(prompt):
    """Nothing but the attributes holds them."""
    import weakref
    gone = weakref.ref(prompt.kv)
    log.clear()
    prompt.kv = None
    assert gone() is None
