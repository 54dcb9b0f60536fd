"""The 4-bit cache's calls on the host: tables and arguments that are refused before anything is launched, and the launches that are made.  No GPU needed."""
import textwrap

from test_host_launches import fake, run  # noqa: F401

SETUP = """
    def create(heads, ctx):
        out = C.c_void_p()
        arr = (hc.hc_kvq_head * len(heads))(*heads)
        return L.hc_kvq_create(ctx, arr, C.byref(out)), out.value
    def table(caps, budget=None, sink=0, recent=0):
        off = row = 0
        heads = []
        for i, cap in enumerate(caps):
            heads.append(hc.hc_kvq_head(off=off, row_off=row, cap=cap, budget=cap if budget is None else budget[i], sink=sink, recent=recent))
            off += 136 * cap
            row += cap
        return heads
    def ctx_of(B, Hkv, G=4, max_ctx=4096):
        cfg = hc.hc_config(B=B, Hq=G * Hkv, Hkv=Hkv, D=128, max_ctx=max_ctx, max_k=8, window=1, metric=0, tau_num=1, tau_den=2, agg=0, window_mode=0)
        out = C.c_void_p()
        assert L.hc_create(C.byref(cfg), C.byref(out)) == 0
        return out.value
    A = lambda k: k << 32
    i32 = lambda *x: (C.c_int32 * len(x))(*x)
    i64 = lambda *x: (C.c_int64 * len(x))(*x)
    def refused(st, want, ctx, text):
        assert st == want and text in L.hc_last_error(ctx).decode(), (st, want, L.hc_last_error(ctx))
        assert fake.fake_log() == b""
"""


def body(s):
    return textwrap.dedent(SETUP) + textwrap.dedent(s)


def test_tables(fake):  # noqa: F811
    run(fake, body("""
        ctx = ctx_of(1, 3)
        def change(i, **kw):
            t = table([64, 16, 4096])
            for k, v in kw.items():
                setattr(t[i], k, v)
            return create(t, ctx)[0]
        assert change(0) == 0
        for kw, text in ((dict(cap=0), "cap 0"), (dict(cap=15), "cap 15"), (dict(cap=-16), "cap"), (dict(cap=4112), "cap 4112")):
            refused(change(2, **kw), hc.HC_ESHAPE, ctx, text)
        for kw, text in ((dict(off=-64), "off"), (dict(off=32), "off"), (dict(row_off=-1), "row_off"), (dict(budget=0), "budget"), (dict(budget=17), "budget"),
                         (dict(sink=-1), "sink"), (dict(recent=-1), "recent"), (dict(sink=2 ** 30 + 1), "sink"), (dict(recent=2 ** 31 - 1), "recent"), (dict(off=64), "overlap"), (dict(row_off=63), "overlap"), (dict(off=0), "overlap")):
            refused(change(1, **kw), hc.HC_EINVAL, ctx, text)
        # a program's sink and recent rows are the same for contexts shorter than they are
        for kw in (dict(sink=4097), dict(recent=4097), dict(sink=2 ** 30, recent=2 ** 30)):
            assert change(1, **kw) == 0, kw
        assert L.hc_kvq_create(ctx, None, C.byref(C.c_void_p())) == hc.HC_EINVAL
        assert L.hc_kvq_create(None, None, None) == hc.HC_ESTATE
        assert L.hc_kvq_destroy(None) == hc.HC_ESTATE
        assert L.hc_kvq_work_bytes(ctx, None) == 0 and L.hc_kvq_work_bytes(None, None) == 0
        st, k = create(table([64, 16, 4096]), ctx)
        assert L.hc_kvq_work_bytes(ctx, k) > 4176 * 16 and L.hc_kvq_work_bytes(ctx_of(1, 3), k) == 0
        assert L.hc_kvq_destroy(k) == 0
        # an address shared by blocks of different heads in any order
        t = table([64, 64, 64]); t[0].off, t[2].off = t[2].off, t[0].off; t[0].row_off, t[2].row_off = t[2].row_off, t[0].row_off
        assert create(t, ctx)[0] == 0
    """))


def test_refused_calls(fake):  # noqa: F811
    run(fake, body("""
        ctx, other = ctx_of(2, 1), ctx_of(2, 1)
        kvq, small = create(table([64, 128]), ctx)[1], create(table([32, 32], [16, 32], 8, 8), ctx)[1]
        tight = create(table([32, 32], [16, 32], 8, 9), ctx)[1]
        foreign = create(table([64, 128]), other)[1]
        rope = hc.hc_rope()
        assert L.hc_rope_init(C.byref(rope), 0, 128, 10000.0, None) == 0
        W = L.hc_kvq_work_bytes(ctx, kvq)
        first, count, off = i32(0, 0), i32(3, 4), i64(0, 8192)
        fake.fake_reset(0)
        ok = dict(ctx=ctx, kvq=kvq, kv=A(1), k_off=off, v_off=off, first=first, count=count, arena=A(2), state=A(3), acc=A(4))
        def store(**kw):
            a = {**ok, **kw}
            return L.hc_kvq_store(a["ctx"], a["kvq"], a["kv"], a["k_off"], a["v_off"], a["first"], a["count"], a["arena"], a["state"], a["acc"], None)
        def load(**kw):
            a = {**ok, **kw}
            return L.hc_kvq_load(a["ctx"], a["kvq"], a["arena"], a["state"], a["first"], a["count"], a["kv"], a["k_off"], a["v_off"], None)
        for call in (store, load):
            assert call(ctx=None) == hc.HC_ESTATE
            for kw, want, text in ((dict(kvq=None), hc.HC_ESTATE, "cache"), (dict(kvq=foreign), hc.HC_ESTATE, "cache"), (dict(kv=None), hc.HC_EINVAL, "null"),
                                   (dict(arena=None), hc.HC_EINVAL, "null"), (dict(state=None), hc.HC_EINVAL, "null"), (dict(first=None), hc.HC_EINVAL, "null"),
                                   (dict(count=None), hc.HC_EINVAL, "null"), (dict(k_off=None), hc.HC_EINVAL, "null"), (dict(arena=A(2) + 32), hc.HC_EINVAL, "64-byte"),
                                   (dict(state=A(3) + 4), hc.HC_EINVAL, "state"), (dict(kv=A(1) + 8), hc.HC_EINVAL, "16-byte"),
                                   (dict(first=i32(-1, 0)), hc.HC_EINVAL, "negative"), (dict(count=i32(1, -1)), hc.HC_EINVAL, "negative"),
                                   (dict(first=i32(4090, 0), count=i32(7, 1)), hc.HC_ESHAPE, "max_ctx"), (dict(k_off=i64(0, 4)), hc.HC_EINVAL, "offsets"),
                                   (dict(v_off=i64(-8, 0)), hc.HC_EINVAL, "offsets")):
                refused(call(**kw), want, ctx, text)
            assert call(count=i32(0, 0)) == 0 and fake.fake_log() == b""
        refused(store(acc=A(4) + 2), hc.HC_EINVAL, ctx, "weights")
        def append(**kw):
            a = {**dict(ctx=ctx, kvq=kvq, rope=C.byref(rope), q=A(1), k=A(2), v=A(3), s=512, kind=0, q_out=A(4), arena=A(5), state=A(6), acc=None), **kw}
            return L.hc_kvq_append(a["ctx"], a["kvq"], a["rope"], a["q"], a["k"], a["v"], a["s"], a["s"], a["s"], a["kind"], a["q_out"], a["arena"], a["state"], a["acc"], None)
        assert append(ctx=None) == hc.HC_ESTATE
        for kw, want, text in ((dict(kvq=foreign), hc.HC_ESTATE, "cache"), (dict(q=None), hc.HC_EINVAL, "null"), (dict(q_out=None), hc.HC_EINVAL, "null"),
                               (dict(rope=None), hc.HC_EINVAL, "null"), (dict(s=12), hc.HC_EINVAL, "strides"), (dict(s=-8), hc.HC_EINVAL, "strides"),
                               (dict(kind=2), hc.HC_EINVAL, "in_type"), (dict(k=A(2) + 4), hc.HC_EINVAL, "aligned"), (dict(arena=None), hc.HC_EINVAL, "null")):
            refused(append(**kw), want, ctx, text)
        def attn(**kw):
            a = {**dict(ctx=ctx, kvq=kvq, arena=A(1), state=A(2), q=A(3), out=A(4), lse=A(5), acc=A(6), decay=0.5, work=A(7), size=W), **kw}
            return L.hc_kvq_attn(a["ctx"], a["kvq"], a["arena"], a["state"], a["q"], a["out"], a["lse"], a["acc"], a["decay"], a["work"], a["size"], None)
        assert attn(ctx=None) == hc.HC_ESTATE
        for kw, want, text in ((dict(kvq=foreign), hc.HC_ESTATE, "cache"), (dict(q=None), hc.HC_EINVAL, "null"), (dict(out=None), hc.HC_EINVAL, "null"),
                               (dict(lse=None), hc.HC_EINVAL, "null"), (dict(work=None), hc.HC_EINVAL, "null"), (dict(q=A(3) + 8), hc.HC_EINVAL, "16-byte"),
                               (dict(out=A(3)), hc.HC_EINVAL, "overlaps"), (dict(out=A(3) - 4080), hc.HC_EINVAL, "overlaps"), (dict(out=A(3) + 2 * 4 * 256 - 16), hc.HC_EINVAL, "overlaps"),
                               (dict(lse=A(5) + 2), hc.HC_EINVAL, "misaligned"), (dict(decay=-0.1), hc.HC_EINVAL, "decay"), (dict(decay=1.5), hc.HC_EINVAL, "decay"),
                               (dict(decay=float("nan")), hc.HC_EINVAL, "decay"), (dict(work=A(7) + 64), hc.HC_EINVAL, "256-byte"), (dict(size=W - 1), hc.HC_EINVAL, "needed"),
                               (dict(state=A(2) + 4), hc.HC_EINVAL, "state")):
            refused(attn(**kw), want, ctx, text)
        def evict(**kw):
            a = {**dict(ctx=ctx, kvq=kvq, arena=A(1), state=A(2), acc=A(3), to=small, ta=A(4), ts=A(5), tc=A(6), kept=A(7), work=A(8), size=W), **kw}
            return L.hc_kvq_evict(a["ctx"], a["kvq"], a["arena"], a["state"], a["acc"], a["to"], a["ta"], a["ts"], a["tc"], a["kept"], a["work"], a["size"], None)
        assert evict(ctx=None) == hc.HC_ESTATE
        for kw, want, text in ((dict(kvq=foreign), hc.HC_ESTATE, "cache"), (dict(to=foreign), hc.HC_ESTATE, "cache"), (dict(acc=None), hc.HC_EINVAL, "null"),
                               (dict(tc=None), hc.HC_EINVAL, "null"), (dict(ts=None), hc.HC_EINVAL, "null"), (dict(work=None), hc.HC_EINVAL, "null"),
                               (dict(ta=A(1) + 64), hc.HC_EINVAL, "overlap"), (dict(ta=A(1) - 64), hc.HC_EINVAL, "overlap"), (dict(ts=A(2) + 8), hc.HC_EINVAL, "overlap"),
                               (dict(tc=A(3) + 4), hc.HC_EINVAL, "overlap"), (dict(to=tight), hc.HC_EINVAL, "budget of 16"), (dict(kept=A(7) + 1), hc.HC_EINVAL, "list"),
                               (dict(size=W - 1), hc.HC_EINVAL, "needed")):
            refused(evict(**kw), want, ctx, text)
        fake.fake_reset(0)
        assert store() == 0 and load() == 0 and append() == 0 and attn() == 0 and evict() == 0
        assert fake.fake_log() != b""
    """))


def test_a_failed_launch_is_reported(fake):  # noqa: F811
    run(fake, body("""
        ctx = ctx_of(1, 2)
        kvq = create(table([1024, 1024]), ctx)[1]
        to = create(table([64, 64]), ctx)[1]
        W = L.hc_kvq_work_bytes(ctx, kvq)
        off = i64(0, 1 << 20)
        calls = [lambda: L.hc_kvq_store(ctx, kvq, A(1), off, off, i32(0), i32(200), A(2), A(3), None, None),
                 lambda: L.hc_kvq_load(ctx, kvq, A(2), A(3), i32(0), i32(200), A(1), off, off, None),
                 lambda: L.hc_kvq_attn(ctx, kvq, A(1), A(2), A(3), A(4), A(5), None, 1.0, A(7), W, None),
                 lambda: L.hc_kvq_evict(ctx, kvq, A(1), A(2), A(3), to, A(4), A(5), A(6), None, A(8), W, None)]
        for call in calls:
            fake.fake_reset(0)
            assert call() == 0
            n = len(log())
            assert n >= 1
            for k in range(1, n + 1):
                fake.fake_reset(k)
                assert call() == hc.HC_EHIP and len(log()) == k - 1
                fake.fake_reset(0)
                assert call() == 0 and len(log()) == n
    """))


def test_launches_of_many_heads(fake):  # noqa: F811
    """64 sequences to a launch where the blocks of each lie evenly apart, else as many as have room for an offset to a head."""
    run(fake, body("""
        ctx = ctx_of(70, 4, max_ctx=128)
        kvq = create(table([64] * 280), ctx)[1]
        even, odd = i64(*[i * 8192 for i in range(280)]), i64(*[i * i * 8192 for i in range(280)])
        for off, launches, per in ((even, 2, 64), (odd, 3, 32)):
            fake.fake_reset(0)
            assert L.hc_kvq_load(ctx, kvq, A(1), A(2), i32(*[0] * 70), i32(*[3] * 70), A(3), even, off, None) == 0
            assert all("kvq_load" in l[0] and l[2] == "4" for l in log()) and [int(l[1]) for l in log()] == ([per] * launches + [70 - per * (launches - 1)])[-launches:]
            fake.fake_reset(0)
            assert L.hc_kvq_load(ctx, kvq, A(1), A(2), i32(*[0] * 70), i32(*[0] * 69 + [2]), A(3), off, even, None) == 0
            assert len(log()) == 1
    """))


def test_launches_by_the_longest_head(fake):  # noqa: F811
    """Attention over heads of little room is one launch, a workgroup to a head; eviction of short heads two launches, of long ones six."""
    run(fake, body("""
        ctx = ctx_of(1, 3, max_ctx=16384)
        for cap, attn, evict in ((256, ["short"], 2), (272, ["short"], 2), (1024, ["short"], 2), (1040, ["attn", "combine"], 2), (8192, ["attn", "combine"], 2),
                                 (8208, ["attn", "combine"], 6)):
            kvq, to = create(table([16, cap, 32]), ctx)[1], create(table([16, 16, 16]), ctx)[1]
            W = L.hc_kvq_work_bytes(ctx, kvq)
            fake.fake_reset(0)
            assert L.hc_kvq_attn(ctx, kvq, A(1), A(2), A(3), A(4), A(5), A(6), 1.0, A(7), W, None) == 0
            assert len(log()) == len(attn) and all(k in l[0] for k, l in zip(attn, log())), log()
            if attn == ["short"]:
                assert log()[0][1] == "3"
            else:
                assert int(log()[0][1]) <= 512 and int(log()[1][1]) == 3 * 4 + 2 + (cap + 1023) // 1024
            fake.fake_reset(0)
            assert L.hc_kvq_evict(ctx, kvq, A(1), A(2), A(3), to, A(4), A(5), A(6), None, A(8), W, None) == 0
            assert len(log()) == evict
    """))
