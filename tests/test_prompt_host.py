"""The host side of the operators in front of the cache: frequencies, refusals, and the launches of a call.  No GPU needed (fake_hip.cpp stands in for the
HIP runtime, in a process of its own)."""
import ctypes as C
import math

import pytest

from paper_2601_13684_amd import binding as hc

from test_host_launches import fake, run  # noqa: F401


def freqs(r):
    return [r.freq[i] for i in range(64)]


@pytest.mark.parametrize("rot,theta", [(128, 10000.0), (64, 500000.0), (8, 1e6), (0, 10000.0)])
def test_plain_frequencies(rot, theta):
    r = hc.hc_rope_init(hc.HC_ROPE_HALF, rot, theta)
    want = [math.exp(-2 * i / rot * math.log(theta)) for i in range(rot // 2)] + [0.0] * (64 - rot // 2)
    assert freqs(r) == pytest.approx(want, rel=1e-14, abs=0)
    assert r.gain == 1.0 and r.eps == pytest.approx(1e-6) and r.q_norm is None and r.k_norm is None and r.rot_dim == rot


def test_fitted_frequencies():
    plain = freqs(hc.hc_rope_init(1, 128, 500000.0))
    lin = freqs(hc.hc_rope_init(1, 128, 500000.0, hc.hc_rope_scaling(kind=hc.HC_ROPE_LINEAR, factor=4.0)))
    assert lin == pytest.approx([f / 4 for f in plain], rel=1e-14)
    base = freqs(hc.hc_rope_init(1, 128, 500000.0, hc.hc_rope_scaling(kind=hc.HC_ROPE_BASE, factor=4.0)))
    assert base[0] == 1.0 and base[63] == pytest.approx(plain[63] / 4, rel=1e-12)      # the fastest stays, the slowest is divided by the factor
    bands = freqs(hc.hc_rope_init(1, 128, 500000.0, hc.hc_rope_scaling(kind=hc.HC_ROPE_BANDS, original=8192, factor=8.0, low=1.0, high=4.0)))
    for f, g in zip(plain, bands):
        wave = 2 * math.pi / f
        if wave < 8192 / 4:
            want = f
        elif wave > 8192:
            want = f / 8
        else:
            s = (8192 / wave - 1) / 3
            want = (1 - s) * f / 8 + s * f
        assert g == pytest.approx(want, rel=1e-12)
    assert bands[0] == plain[0] and bands[63] == plain[63] / 8


@pytest.mark.parametrize("args,scaling,status", [
    ((2, 128, 1e4), None, hc.HC_EINVAL), ((0, 12, 1e4), None, hc.HC_ESHAPE), ((0, 136, 1e4), None, hc.HC_ESHAPE), ((0, -8, 1e4), None, hc.HC_ESHAPE),
    ((0, 128, 0.0), None, hc.HC_EINVAL), ((0, 128, -1.0), None, hc.HC_EINVAL), ((0, 128, math.nan), None, hc.HC_EINVAL), ((0, 128, math.inf), None, hc.HC_EINVAL),
    ((0, 128, 1e-300), None, hc.HC_EINVAL),
    ((0, 128, 1e4), dict(kind=3, factor=2.0), hc.HC_EINVAL), ((0, 128, 1e4), dict(kind=0, factor=0.5), hc.HC_EINVAL),
    ((0, 128, 1e4), dict(kind=0, factor=math.nan), hc.HC_EINVAL), ((0, 128, 1e4), dict(kind=2, factor=2.0, low=1.0, high=1.0, original=10), hc.HC_EINVAL),
    ((0, 128, 1e4), dict(kind=2, factor=2.0, low=1.0, high=4.0, original=0), hc.HC_EINVAL),
    ((0, 128, 1e4), dict(kind=2, factor=2.0, low=1.0, high=math.inf, original=9), hc.HC_EINVAL),
])
def test_refused_ropes(args, scaling, status):
    with pytest.raises(hc.HcError) as e:
        hc.hc_rope_init(*args, hc.hc_rope_scaling(**scaling) if scaling else None)
    assert e.value.status == status


def test_struct_sizes_and_null_arguments():
    assert C.sizeof(hc.hc_rope) == 4 * 4 + 2 * 8 + 64 * 8 and C.sizeof(hc.hc_rope_scaling) == 2 * 4 + 3 * 8
    L = hc.lib()
    assert L.hc_rope_init(None, 0, 128, 1e4, None) == hc.HC_EINVAL
    assert L.hc_prefill_attn_work_bytes(None) == 0
    assert L.hc_prefill_attn(*([None] * 10 + [0, None])) == hc.HC_ESTATE
    assert L.hc_prefill_rope(*([None] * 5 + [0] * 4 + [None] * 7)) == hc.HC_ESTATE
    assert L.hc_append_rope(*([None] * 6 + [0] * 4 + [None] * 4)) == hc.HC_ESTATE


CALLS = '''
def ints(v):
    return (C.c_int32 * len(v))(*v)
def longs(v):
    return (C.c_int64 * len(v))(*v)
def cfg(B, Hkv, G, max_ctx=4096):
    c = hc.hc_config(B=B, Hq=Hkv * G, Hkv=Hkv, D=128, max_ctx=max_ctx, max_k=8, window=1, metric=0, tau_num=1, tau_den=2, agg=0, window_mode=0)
    out = C.c_void_p()
    assert L.hc_create(C.byref(c), C.byref(out)) == 0
    return out.value
A = 1 << 20                                        # an address that nothing reads, 1 MiB-aligned
def attn(ctx, n, **kw):
    """n: sequences times KV heads."""
    a = dict(q=A, kv=A, k=[8 * i for i in range(n)], v=[8 * i for i in range(n)], first=[0], count=[5], out=A, lse=A, work=A, bytes=1 << 40)
    a.update(kw)
    arr = lambda f, x: None if x is None else f(x)
    return L.hc_prefill_attn(ctx, a["q"], a["kv"], arr(longs, a["k"]), arr(longs, a["v"]), arr(ints, a["first"]), arr(ints, a["count"]), a["out"], a["lse"],
                             a["work"], a["bytes"], None)
rope0 = hc.hc_rope()
assert L.hc_rope_init(C.byref(rope0), 0, 128, 1e4, None) == 0
def rope_with(**kw):
    r = hc.hc_rope.from_buffer_copy(rope0)
    for k, v in kw.items():
        if k == "freq0":
            r.freq[0] = v
        else:
            setattr(r, k, v)
    return r
def rope(ctx, n, **kw):
    a = dict(r=rope0, q=A, k=A, v=A, qs=4096, ks=1024, vs=1024, type=0, first=[0], count=[5], out=A, kv=A, ko=[8 * i for i in range(n)], vo=[8 * i for i in range(n)])
    a.update(kw)
    arr = lambda f, x: None if x is None else f(x)
    return L.hc_prefill_rope(ctx, None if a["r"] is None else C.byref(a["r"]), a["q"], a["k"], a["v"], a["qs"], a["ks"], a["vs"], a["type"], arr(ints, a["first"]),
                             arr(ints, a["count"]), a["out"], a["kv"], arr(longs, a["ko"]), arr(longs, a["vo"]), None)
def append(ctx, lay, **kw):
    a = dict(r=rope0, q=A, k=A, v=A, qs=4096, ks=1024, vs=1024, type=0, out=A, arena=A, tier=A)
    a.update(kw)
    return L.hc_append_rope(ctx, lay, None if a["r"] is None else C.byref(a["r"]), a["q"], a["k"], a["v"], a["qs"], a["ks"], a["vs"], a["type"], a["out"], a["arena"],
                            a["tier"], None)
'''


def test_refused_calls(fake):  # noqa: F811
    run(fake, CALLS + '''
E, S, ST = hc.HC_EINVAL, hc.HC_ESHAPE, hc.HC_ESTATE
ctx = cfg(1, 2, 4)
fake.fake_reset(0)
need = L.hc_prefill_attn_work_bytes(ctx)
assert need > 0
for kw, want in [(dict(q=None), E), (dict(kv=None), E), (dict(k=None), E), (dict(v=None), E), (dict(first=None), E), (dict(count=None), E), (dict(out=None), E),
                 (dict(work=None), E), (dict(bytes=need - 1), E), (dict(q=A + 8), E), (dict(kv=A + 8), E), (dict(out=A + 8), E), (dict(lse=A + 2), E), (dict(work=A + 128), E),
                 (dict(first=[-1]), E), (dict(count=[-1]), E), (dict(first=[4092]), S), (dict(count=[4097]), S), (dict(first=[2**31 - 1], count=[2**31 - 1]), S),
                 (dict(k=[4, 8]), E), (dict(v=[0, -8]), E)]:
    assert attn(ctx, 2, **kw) == want, (kw, L.hc_last_error(ctx))
    assert b"hc_prefill_attn" in L.hc_last_error(ctx), kw
nan = float("nan")
for kw, want in [(dict(r=None), E), (dict(q=None), E), (dict(k=None), E), (dict(v=None), E), (dict(out=None), E), (dict(kv=None), E), (dict(ko=None), E), (dict(first=None), E),
                 (dict(q=A + 8), E), (dict(k=A + 8), E), (dict(v=A + 8), E), (dict(out=A + 8), E), (dict(kv=A + 8), E), (dict(qs=4100), E), (dict(ks=-8), E), (dict(vs=1 << 33), E),
                 (dict(type=2), E), (dict(type=-1), E), (dict(first=[4092]), S), (dict(count=[-2]), E), (dict(ko=[4, 8]), E),
                 (dict(r=rope_with(layout=2)), E), (dict(r=rope_with(rot_dim=12)), S), (dict(r=rope_with(rot_dim=136)), S), (dict(r=rope_with(eps=-1.0)), E), (dict(r=rope_with(eps=nan)), E),
                 (dict(r=rope_with(gain=nan)), E), (dict(r=rope_with(q_norm=A + 4)), E), (dict(r=rope_with(k_norm=A + 4)), E), (dict(r=rope_with(freq0=nan)), E), (dict(r=rope_with(freq0=1e7)), E)]:
    assert rope(ctx, 2, **kw) == want, (kw, L.hc_last_error(ctx))
    assert b"hc_prefill_rope" in L.hc_last_error(ctx), kw
lctx = context(500, 30)
lay = layer(lctx, 500, 30)
fake.fake_reset(0)
full = append(lctx, lay)                            # no room to grow
assert full == S and b"hc_append_rope" in L.hc_last_error(lctx)
assert append(ctx, lay) == ST and b"hc_append_rope" in L.hc_last_error(ctx)
many = cfg(1, 129, 1)
fake.fake_reset(0)
assert attn(many, 129) == S and rope(many, 129) == S
big = cfg(2, 1, 8, 1 << 24)
fake.fake_reset(0)
assert attn(big, 2, first=[0, 0], count=[1 << 24, 1 << 24]) == 0 and len(log()) == 1           # 2^28 rows of queries
n = 1 << 24
more = cfg(3, 1, 1, n)
fake.fake_reset(0)
assert attn(more, 3, first=[0] * 3, count=[n, n, 1]) == S and rope(more, 3, first=[0] * 3, count=[n, 1, n]) == S and not log()      # 2^25 tokens
wide = cfg(9, 4, 8, n)
fake.fake_reset(0)
assert attn(wide, 36, first=[0] * 9, count=[n] + [1] + [0] * 7) == S and rope(wide, 36, first=[0] * 9, count=[0] * 8 + [n]) == 0      # 2^29 rows
huge = cfg(64, 1, 8, 1 << 24)
fake.fake_reset(0)
assert attn(huge, 64, first=[0] * 64, count=[1 << 24] * 64) == S
assert not log(), log()
''')


def test_refused_appends(fake):  # noqa: F811
    run(fake, CALLS + '''
c = hc.hc_config(B=1, Hq=8, Hkv=2, D=128, max_ctx=1024, max_k=64, window=1, metric=0, tau_num=1, tau_den=2, agg=0, window_mode=0)
out = C.c_void_p()
assert L.hc_create(C.byref(c), C.byref(out)) == 0
ctx = out.value
descs = (hc.hc_head_desc * 2)(hc.hc_head_desc(k_off=0, v_off=1 << 20, ctx=500, len=500, role=0, rep=-1, cap=510),
                              hc.hc_head_desc(k_off=1 << 21, v_off=1 << 22, tier_off=0, ctx=500, len=60, role=1, rep=0, sink=4, recent=20, cap=510))
lay = C.c_void_p()
assert L.hc_layer_create(ctx, descs, C.byref(lay)) == 0, L.hc_last_error(ctx)
fake.fake_reset(0)
E, S = hc.HC_EINVAL, hc.HC_ESHAPE
for kw, want in [(dict(r=None), E), (dict(q=None), E), (dict(k=None), E), (dict(v=None), E), (dict(out=None), E), (dict(arena=None), E), (dict(tier=None), E), (dict(arena=A + 8), E),
                 (dict(tier=A + 8), E), (dict(q=A + 4), E), (dict(out=A + 8), E), (dict(qs=4), E), (dict(type=5), E), (dict(r=rope_with(rot_dim=4)), S)]:
    assert append(ctx, lay, **kw) == want, (kw, L.hc_last_error(ctx))
    assert b"hc_append_rope" in L.hc_last_error(ctx), kw
    assert L.hc_layer_context(lay, 0) == 500
assert not log()
fake.fake_reset(1)                                  # a launch that fails leaves the lengths where they were
assert append(ctx, lay) == hc.HC_EHIP and L.hc_layer_context(lay, 0) == 500
fake.fake_reset(0)
assert append(ctx, lay) == 0 and L.hc_layer_context(lay, 0) == 501
assert len(log()) == 1 and log()[0][1] == "2"
''')


def test_launches(fake):  # noqa: F811
    run(fake, CALLS + '''
import random
ctx = cfg(1, 2, 4)
fake.fake_reset(0)
assert attn(ctx, 2, count=[0]) == 0 and rope(ctx, 2, count=[0], q=None, out=None) == 0 and not log()
assert rope(ctx, 2, count=[9]) == 0 and len(log()) == 1
# seventy sequences of two heads, forty of eight: more than a launch's arguments hold, so that the table goes to the work buffer first
for B, H, n in ((64, 2, 1), (65, 1, 2), (70, 2, 2), (40, 8, 3)):
    c = cfg(B, H, 4)
    fake.fake_reset(0)
    assert rope(c, B * H, first=[0] * B, count=[3] * B) == 0 and len(log()) == n, log()
    fake.fake_reset(0)
    assert attn(c, B * H, first=[0] * B, count=[3] * B) == 0
    names = [l[0] for l in log()]
    assert len([x for x in names if "prompt_attn_kernel" in x]) == 1 and len([x for x in names if "prompt_table_kernel" in x]) == (n if n > 1 else 0), names
fake.fake_reset(1)
assert attn(c, B * H, first=[0] * B, count=[3] * B) == hc.HC_EHIP and not log()
''')


def test_pieces_fit_the_work_buffer(fake):  # noqa: F811
    """Over random batches: every plan has room for its pieces' rows in the work buffer (the call looks again before it launches, and would refuse)."""
    run(fake, CALLS + '''
import random, re
rng = random.Random(5)
split = 0
for trial in range(600):
    B, H, G = rng.choice([1, 1, 2, 3, 9, 30, 64, 200]), rng.choice([1, 2, 8]), rng.choice([1, 2, 4, 8])
    c = cfg(B, H, G, 1 << 24)
    size = rng.choice([1, 10, 1000])
    count = [rng.randint(0, size) for _ in range(B)]
    first = [int(2 ** rng.uniform(0, rng.choice([3, 12, 23.9]))) for _ in range(B)]
    fake.fake_reset(0)
    assert attn(c, B * H, first=first, count=count) == 0
    names = [(l[0], int(l[1])) for l in log()]
    split += any("join" in n for n, _ in names)
    assert bool(names) == (sum(count) > 0)
    if not names:
        continue
    (units, rows), = [(u, 128 // int(re.search("prompt_attn_kernelILi[0-9]ELi([12])E", n)[1])) for n, u in names if "prompt_attn" in n]
    tiles = sum((n * G + rows - 1) // rows for n in count) * H
    assert units >= tiles and (any("join" in n for n, _ in names) or units == tiles), (units, tiles)
assert split > 100, split
''')
