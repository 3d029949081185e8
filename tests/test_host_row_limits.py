"""Launches of the calls on a batch's rows at the ends of their ranges, on the stand-in HIP runtime (no GPU; tests/test_host_dispatch.py)."""
import textwrap

import pytest

from tests.test_host_dispatch import CXX, run, runtime  # noqa: F401
from tests.test_host_row_calls import CALLS

pytestmark = pytest.mark.skipif(CXX is None, reason="needs g++")


def test_add_norm_launches_fewer_threads_than_a_launch_may_have(runtime):  # noqa: F811
    run(runtime, textwrap.dedent(CALLS) + textwrap.dedent("""
        import re
        p, f = make_pool(), make_pool(kv_dtype=B.F32)
        for pool, res in ((p, B.BF16), (p, B.F32), (f, B.F32)):
            for n in (1, 1 << 14, 1 << 18, (1 << 22) - 1, 1 << 22):
                for width in (512, 1024, 2048, 4096, 8192, 8200, 16384, 16392, 32768):
                    (name, grid, lds), = launched(lambda: norm(pool, n=n, width=width, bs=width, rs=width, residual_dtype=res))
                    waves, pieces = map(int, re.search(r"Li(\\d+)ELi(\\d+)E", name).groups())
                    assert "add_norm_kernel" in name and grid[1:] == (1, 1)
                    assert grid[0] * max(256, 64 * waves) < 1 << 32, (n, width, name, grid)
                    assert waves * pieces * 512 >= width and grid[0] * (4 // waves if waves < 4 else 1) >= n
    """))


def test_group_adapters_of_batches_beyond_32_bits(runtime):  # noqa: F811
    """Lists whose sums may be beyond 32 bits are made by a kernel of their own."""
    run(runtime, textwrap.dedent(CALLS) + textwrap.dedent("""
        p = make_pool(max_requests=3000)
        for n, max_rows, start, capped in ((2, 1 << 27, OFFS, False), (31, 1 << 27, OFFS, False), (32, 1 << 27, OFFS, True), (32, (1 << 27) - 1, OFFS, False),
                                           (3000, 1431655, OFFS, False), (3000, 1431656, OFFS, True), (3000, 1 << 27, None, False)):
            (name, grid, lds), = launched(lambda: group(p, n=n, max_rows=max_rows, start=start, max_items=(max_rows >> 6) + 4))
            assert "group_adapters_kernel" in name and ("Lb1E" in name) == capped, (n, max_rows, name)
    """))


def test_adapt_rows_takes_what_the_header_says(runtime):  # noqa: F811
    run(runtime, textwrap.dedent(CALLS) + textwrap.dedent("""
        p = make_pool()
        for cols, rank in (((64, 32), 16), ((4096, 512, 520 - 8), 16), ((16,), 256), ((1040, 16, 16, 16), 256)):
            pieces = max(sum(-(-c // 512) for c in cols), -(-len(cols) * rank // 64))
            most = ((1 << 24) - 1) // pieces // 32 * 32
            ad = make(part_cols=cols, rank=rank)
            wide = dict(n=1 << 27, ad=ad, bs=sum(cols), ys=sum(cols))
            assert len(launched(lambda: adapt(p, max_items=most, **wide))) == 2 and p.odma_adapt_scratch_bytes(ad, most)
            assert refused(adapt, p, max_items=most + 1, **wide), (cols, rank)
        adapt(p, ad=make(width=32768), xs=32768)
        assert refused(adapt, p, ad=make(width=32776), xs=32776) and refused(adapt, p, n=(1 << 27) + 1)
    """))


def test_adapt_rows_of_fp8_pools_launch_as_those_of_bf16_pools(runtime):  # noqa: F811
    """Their rows are bf16 too: the same bytes to a line and past the caches."""
    run(runtime, textwrap.dedent(CALLS) + textwrap.dedent("""
        p, q = make_pool(), make_pool(kv_dtype=B.FP8)
        for n, items, cols, rank in ((100, 6, (64, 32), 16), (100000, 1590, (3584, 512, 512), 16), (100000, 1590, (64, 4544), 16), (100000, 1590, (4672,), 64),
                                     (20000, 4000, (192,), 16), (9000, 8000, (320,), 8)):
            one, two = (launched(lambda: adapt(pool, n=n, max_items=items, bs=sum(cols), ys=sum(cols), ad=make(part_cols=cols, rank=rank))) for pool in (p, q))
            assert one == two, (one, two)
    """))
