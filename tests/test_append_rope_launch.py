"""The decode token's workgroups: a row of threads for K, V and every query head, of no more threads than the kernel is built for.  No GPU needed."""
from test_host_launches import fake, run  # noqa: F401
from test_kernel_resources import kernels, of  # noqa: F401


def test_threads_for_every_group(fake, kernels):  # noqa: F811
    built = {k["threads"] for k in of(kernels, "append_rope_kernel").values()}
    run(fake, '''
rope = hc.hc_rope()
assert L.hc_rope_init(C.byref(rope), 0, 128, 1e4, None) == 0
A = 1 << 20
most = 0
for G in range(1, 20):
    cfg = hc.hc_config(B=2, Hq=3 * G, Hkv=3, D=128, max_ctx=1024, max_k=8, window=1, metric=0, tau_num=1, tau_den=2, agg=0, window_mode=0)
    ctx, lay = C.c_void_p(), C.c_void_p()
    st = L.hc_create(C.byref(cfg), C.byref(ctx))
    assert (st == 0) == (G in (1, 2, 4, 8)) and st in (0, hc.HC_ESHAPE), (G, st)
    if st:
        continue
    descs = (hc.hc_head_desc * 6)(*[hc.hc_head_desc(k_off=i << 21, v_off=(2 * i + 1) << 20, ctx=500, len=500, role=0, rep=-1, cap=510) for i in range(6)])
    assert L.hc_layer_create(ctx, descs, C.byref(lay)) == 0, L.hc_last_error(ctx)
    fake.fake_reset(0)
    assert L.hc_append_rope(ctx, lay, C.byref(rope), A, A, A, 4096, 1024, 1024, 0, A, A, None, None) == 0
    (name, x, y, z, threads, *_), = log()
    assert "append_rope_kernel" in name and int(x) == 6 and 16 * (G + 2) <= int(threads) < 16 * (G + 2) + 64 and int(threads) %% 64 == 0, log()
    most = max(most, int(threads))
assert {most} == %r, most
''' % built)
