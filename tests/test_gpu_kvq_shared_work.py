"""A work buffer that two caches held in 4 bits share, and streams.  Run with `-m gpu` on an MI355X."""
import pytest
import torch

import kvq_util as U
from paper_2601_13684_amd import binding as hc
from paper_2601_13684_amd import runtime as R

pytestmark = pytest.mark.gpu
DEV, D = U.DEV, U.D


@pytest.mark.parametrize("made_there", [False, True])
@pytest.mark.parametrize("owned", [True, False])
def test_both_dropped_while_the_other_stream_works(made_there, owned):
    """The buffer's owner has never been on the side stream, whose queue is long.  Both caches are dropped: as long as that stream is not through, no other tensor has the buffer's
    place, and what is written over it afterwards reaches no result."""
    B, Hkv, G, n = 1, 2, 4, 20000
    ctx = R.Context(hc.hc_config(B=B, Hq=Hkv * G, Hkv=Hkv, D=D, max_ctx=20032, max_k=8, window=1, metric=0, tau_num=1, tau_den=2, agg=0, window_mode=0), DEV)
    table, to = R.QuantTable(ctx, [n] * Hkv), R.QuantTable(ctx, [512] * Hkv, [500] * Hkv, 4, 50)
    g = torch.Generator(device=DEV)
    g.manual_seed(2)
    codes = torch.randint(0, 256, (table.nbytes,), generator=g, dtype=torch.uint8, device=DEV)
    for h in table.heads:                        # (scales of about 1)
        for v in (0, 1):
            at = h.off + 68 * h.cap * v + 64 * h.cap
            codes[at:at + 4 * h.cap] = 126
    q = torch.randn((B, Hkv * G, D), generator=g, device=DEV).to(torch.bfloat16)
    side, busy = torch.cuda.Stream(), torch.empty((1 << 28,), dtype=torch.float32, device=DEV)
    size, out, lse = table.work_bytes(), torch.empty((B, Hkv * G, D), device=DEV), torch.empty((B, Hkv * G), device=DEV)

    def use(stream):
        owner = R.QuantCache(table).work if owned else torch.empty((size,), dtype=torch.uint8, device=DEV)
        with torch.cuda.stream(side if made_there else torch.cuda.current_stream()):
            cache = R.QuantCache(table, work=owner)
        cache.arena.copy_(codes)
        cache.state.copy_(torch.tensor([[n, n]] * Hkv, dtype=torch.int32))
        small = R.QuantCache(to)
        torch.cuda.synchronize()
        if stream is not None:
            with torch.cuda.stream(stream):
                for _ in range(60):
                    busy.fill_(1.0)              # milliseconds
        cache.attn(q, 1.0, out, lse, stream=stream)
        cache.evict(small, stream=stream)
        return owner.data_ptr(), small
    _, small = use(None)
    torch.cuda.synchronize()
    want = [t.clone() for t in (out, lse, small.acc, small.state)]
    out.zero_(), lse.zero_()
    del small
    torch.cuda.synchronize()
    torch.empty((1,), device=DEV)
    held = torch.cuda.memory_allocated()
    place, small = use(side)                     # (owner and cache are gone)
    noise = [torch.full((size,), 255, dtype=torch.uint8, device=DEV) for _ in range(4)]
    there = [t.data_ptr() for t in noise]
    assert not side.query()                      # (else nothing is shown)
    assert place not in there
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((out, lse, small.acc, small.state), want))
    del noise, small
    torch.cuda.synchronize()
    torch.empty((1,), device=DEV)                # (the allocator looks through what it keeps when it is asked)
    assert torch.cuda.memory_allocated() == held                  # (given back then)
    table.close()
    to.close()
    ctx.close()
