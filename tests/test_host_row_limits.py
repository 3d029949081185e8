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
