"""Which kernels attention over the cache held in 4 bits launches by the number of heads, and how many of their workgroups a compute unit holds.  No GPU needed."""
import re

import pytest

from test_host_launches import fake, run  # noqa: F401
from test_kernel_resources import CU_LDS, SIMD_REGS, kernels  # noqa: F401
from test_kvq_host import body

FIT = 3             # workgroups of 512 threads of the join


@pytest.mark.parametrize("G", [1, 2, 4, 8])
def test_the_join_by_the_number_of_query_heads(fake, G):  # noqa: F811
    """More query heads than 256 compute units hold workgroups of 512 threads: 128 threads each."""
    run(fake, body(f"""
        G, most = {G}, 256 * {FIT} // {G}
        for n in (1, most - 1, most, most + 1, 1024 // G, 1024 // G + 1, 4096):
            ctx = ctx_of(1 if n % 2 else 2, n if n % 2 else n // 2, G, max_ctx=2048)
            kvq = create(table([1040] + [16] * (n - 1)), ctx)[1]
            W = L.hc_kvq_work_bytes(ctx, kvq)
            for acc, chunks in ((None, 0), (A(6), n + 1)):
                fake.fake_reset(0)
                assert L.hc_kvq_attn(ctx, kvq, A(1), A(2), A(3), A(4), A(5), acc, 1.0, A(7), W, None) == 0
                name, x, y, z, threads = log()[1][:5]
                assert "combine" in name and int(threads) == (512 if n <= most else 128) and int(x) == n * G + chunks, (n, log())
    """))


def held(k):
    """Workgroups that a compute unit holds, by registers and by LDS."""
    waves = k["threads"] // 64
    return min(4 * min(8, SIMD_REGS // k["regs"]) // waves, CU_LDS // max(1, k["lds"]))


def test_workgroups_that_fit(kernels):  # noqa: F811
    join = {m: k for name, k in kernels.items() for m in re.findall(r"kvq_combine_kernelILi(\d)ELi512E", name)}
    assert sorted(join) == ["1", "2", "4", "8"] and all(held(k) == FIT and k["scratch"] == 0 for k in join.values()), join
    short = {m: k for name, k in kernels.items() for m in re.findall(r"kvq_attn_short_kernelILi(\d)ELb(\d)ELi(\d)E", name)}
    assert len(short) == 24
    for (g, weights, buffers), k in short.items():
        want = {"4": 1, "2": 2, "1": 4 if weights == "0" and g != "8" else 3}[buffers]
        assert held(k) == want and k["scratch"] == 0, (g, weights, buffers, k)
    split = {m: k for name, k in kernels.items() for m in re.findall(r"kvq_attn_kernelILi(\d)ELb(\d)E", name)}
    assert len(split) == 8 and all(held(k) >= 2 and k["scratch"] == 0 for k in split.values()), split
