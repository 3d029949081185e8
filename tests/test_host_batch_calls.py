"""Refusals and launches of the calls that prepare a batch and of attention over shared prefixes, on the stand-in HIP runtime
(no GPU; tests/test_host_dispatch.py): what a call refuses launches nothing, what it takes launches what is written here."""
import pytest

from tests.test_host_dispatch import CXX, run, runtime  # noqa: F401

pytestmark = pytest.mark.skipif(CXX is None, reason="needs g++")

CALLS = """
    START, POFF, PLEN, SLOT, POS = ((i + 20) << 32 for i in range(5))

    def tables(p, n=4, lengths=LENS, n_new=None, offsets=OFFS, np_=1, start=START, poff=POFF, plen=PLEN, bt=TABLE, stride=8,
               rows=16, row_start=Q, pos=POS, slot=SLOT):
        p.odma_build_tables(n, lengths, n_new, offsets, np_, start, poff, plen, bt, stride, rows, row_start, pos, slot, 0)

    def rows(p, layer=0, n=5, prep=None, q=Q, qs=1024, k=K, ks=1024, v=V, vs=1024, slot=SLOT, pos=POS, out=OUT, **kw):
        args = dict(rot_dim=32, inv_freq=NEW)
        args.update(kw)
        p.odma_append_qkv(layer, n, B.make_qk_prep(**args) if prep is None else prep, q, qs, k, ks, v, vs, slot, pos, out, 0)

    def shared(p, layer=0, n=4, q=Q, np_=1, start=START, poff=POFF, plen=PLEN, offsets=OFFS, lengths=LENS, bt=None, stride=0, out=OUT):
        p.odma_decode_attention_shared(layer, n, q, np_, start, poff, plen, offsets, lengths, bt, stride, out, 0)

    def refused(call, *a, **kw):
        at = hip.fake_launches()
        try:
            call(*a, **kw)
        except B.OdmaError as e:
            assert e.code == B.INVALID_ARG, e
            assert hip.fake_launches() == at
            return True
        return False

    def names(call):
        return [name for name, grid, lds in launched(call)]
"""


def go(runtime, code):  # noqa: F811
    import textwrap
    run(runtime, textwrap.dedent(CALLS) + textwrap.dedent(code))


def test_tables(runtime):  # noqa: F811
    go(runtime, """
        p = make_pool(max_requests=2000)
        for bad in (dict(n=-1), dict(n=2001), dict(lengths=None), dict(offsets=None), dict(stride=0), dict(rows=-1), dict(np_=-1),
                    dict(np_=5), dict(start=None), dict(poff=None), dict(plen=None),
                    dict(bt=None, row_start=None, pos=None, slot=None)):
            assert refused(tables, p, **bad), bad
        assert launched(lambda: tables(p, n=0)) == []
        one = launched(lambda: tables(p))
        assert len(one) == 1 and "build_tables_kernel" in one[0][0] and one[0][1] == (4, 1, 1)
        assert launched(lambda: tables(p, np_=0, start=None, poff=None, plen=None, bt=None, stride=0))[0][1] == (4, 1, 1)
        # long rows are dealt out, many requests share work-groups; up to 1024 work-groups
        assert launched(lambda: tables(p, n=1, rows=1 << 20))[0][1] == (1, 1024, 1)
        assert launched(lambda: tables(p, n=2000, stride=4096))[0][1] == (1000, 1, 1)
        hip.fake_fail_launch(0)
        assert fails(lambda: tables(p))
        cfg, keep = B.make_config(n_layers=1, n_q_heads=4, n_kv_heads=2, head_dim=64, kv_dtype=B.BF16, out_dtype=B.BF16, main_tokens=64,
                                  safety_tokens=64, large_cap=64, boundaries=(64,), quantiles=((1, 2),), max_requests=4)
        bare = B.Pool(cfg, keep)                                  # allocator only
        assert refused(tables, bare) and refused(rows, bare) and refused(shared, bare)
    """)


def test_rows(runtime):  # noqa: F811
    go(runtime, """
        p = make_pool()
        for bad in (dict(layer=-1), dict(layer=1), dict(n=-1), dict(q=None), dict(k=None), dict(v=None), dict(slot=None), dict(out=None),
                    dict(q=Q + 8), dict(k=K + 2), dict(v=V + 4), dict(out=OUT + 8), dict(qs=1028), dict(ks=12), dict(vs=-8),
                    dict(q_weight=Q + 2), dict(k_weight=Q + 8), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")),
                    dict(rot_dim=-8), dict(rot_dim=136), dict(rot_dim=20), dict(inv_freq=None), dict(pos=None), dict(n_axes=0),
                    dict(n_axes=5), dict(n_axes=2, axis=[0, 1, 2]), dict(n=1 << 40), dict(n=(1 << 27) + 1)):
            assert refused(rows, p, **bad), bad
        prep = B.make_qk_prep(rot_dim=32, inv_freq=NEW)
        prep.rot_pairs = 2
        assert refused(rows, p, prep=prep)
        assert B.lib.odma_append_qkv(p._h, 0, 1, None, Q, 0, K, 0, V, 0, SLOT, POS, OUT, None) == B.INVALID_ARG
        for bad in ([0] * 129, [-1], [256]):
            try:
                B.make_qk_prep(axis=bad)
                assert False
            except ValueError:
                pass
        assert launched(lambda: rows(p, n=0)) == []
        # pairs behind the last that turns may name any axis; nothing turns: neither frequencies nor positions
        rows(p, axis=[0] * 16 + [7])
        rows(p, rot_dim=0, inv_freq=None, pos=None)
        # one row: a work-group for each of the 8 + 2 + 2 heads; rounds of 1024 work-groups: 16 rows each, all heads; the rows
        # behind them dealt out again
        assert launched(lambda: rows(p, n=1))[0][1] == (12, 1, 1)
        assert launched(lambda: rows(p, n=16 * 1024))[0][1] == (1024, 1, 1)
        assert launched(lambda: rows(p, n=16 * 1024 + 1))[0][1] == (1024 + 12, 1, 1)
        assert launched(lambda: rows(p, n=16 * (2048 + 300)))[0][1] == (2048 + 4 * 300, 1, 1)
        assert launched(lambda: rows(p, n=16 * 300))[0][1] == (4 * 300, 1, 1)
        assert launched(lambda: rows(p, n=1 << 27))[0][1] == (1 << 23, 1, 1)
        for kv, d in ((B.F32, 32), (B.F32, 256), (B.BF16, 96), (B.FP8, 128)):
            assert "append_qkv_kernel" in names(lambda: rows(make_pool(kv_dtype=kv, head_dim=d)))[0]
        assert refused(rows, make_pool(kv_dtype=B.F32), qs=1026)
        rows(make_pool(kv_dtype=B.F32), qs=1028)
        hip.fake_fail_launch(0)
        assert fails(lambda: rows(p))
    """)


def test_shared(runtime):  # noqa: F811
    go(runtime, """
        p = make_pool()
        for bad in (dict(layer=-1), dict(layer=1), dict(n=-1), dict(n=4097), dict(n=1025), dict(q=None), dict(lengths=None), dict(out=None),
                    dict(offsets=None), dict(bt=TABLE, stride=0), dict(np_=-1), dict(np_=5), dict(start=None), dict(plen=None),
                    dict(poff=None)):
            assert refused(shared, p, **bad), bad
        for kw in (dict(kv_dtype=B.F32), dict(head_dim=96), dict(decode_kernel=B.KERNEL_VALU), dict(sm_scale=-0.1)):
            assert refused(shared, make_pool(**kw)), kw
        assert launched(lambda: shared(p, n=0)) == []
        names_of = names(lambda: shared(p))
        assert "shared_parts_kernel" in names_of[0] and len(names_of) <= 2
        assert names(lambda: shared(p, bt=TABLE, stride=8, poff=None, offsets=None))
        # without prefixes: a decode call
        plain = launched(lambda: decode(p, 4))
        assert launched(lambda: shared(p, np_=0, start=None, poff=None, plen=None)) == plain
        # a plan that decode calls reuse survives
        decode(p, 4)
        reusing = launched(lambda: decode(p, 4, B.REUSE_PLAN))
        shared(p)
        assert launched(lambda: decode(p, 4, B.REUSE_PLAN)) == reusing
        # two work-groups for every compute unit, fewer where the workspace has little room: 8192 columns per query head hold two
        # for each request and head, for each work-group up to 128 and a group of heads for each of its waves, and a record of each request
        for n, hq, hkv in ((1024, 28, 4), (1024, 8, 2), (1024, 1, 1), (3, 2, 1), (4, 16, 1)):
            grid = launched(lambda: shared(make_pool(hq=hq, hkv=hkv), n=n))[0][1]
            used = 2 * n * hq + grid[0] * (min(128, (n * hq // hkv + 15) // 16 * 16) + 4 * hq // hkv)
            assert grid[0] % 8 == 0 and 8 <= grid[0] <= 512 and grid[1:] == (1, 1) and used + n // 8 <= 8192 * hq, (n, hq, grid)
        for kv, d in ((B.BF16, 64), (B.FP8, 128)):
            shared(make_pool(kv_dtype=kv, head_dim=d))
        hip.fake_fail_launch(0)
        assert fails(lambda: shared(p))
    """)


def test_a_call_without_prefixes_leaves_no_plan_to_reuse(runtime):  # noqa: F811
    """It plans for its own lengths, in the same place: a decode call of as many requests that asks for its earlier plan plans again."""
    go(runtime, """
        kernel = lambda call: [hip.fake_name(i).decode() for at in [hip.fake_launches()] for _ in [call()] for i in range(at, hip.fake_launches())]
        for paged in (False, True):
            p = make_pool()
            planning = kernel(lambda: decode(p, 4, paged=paged))
            reusing = kernel(lambda: decode(p, 4, B.REUSE_PLAN, paged))
            assert planning != reusing
            shared(p, np_=0, start=None, poff=None, plen=None, **(dict(bt=TABLE, stride=8, offsets=None) if paged else {}))
            assert kernel(lambda: decode(p, 4, B.REUSE_PLAN, paged)) == planning
            assert kernel(lambda: decode(p, 4, B.REUSE_PLAN, paged)) == reusing
            shared(p)
            assert kernel(lambda: decode(p, 4, B.REUSE_PLAN, paged)) == reusing
            # one that is refused or has no requests changes nothing
            assert refused(shared, p, np_=0, q=None)
            shared(p, np_=0, n=0)
            assert kernel(lambda: decode(p, 4, B.REUSE_PLAN, paged)) == reusing
    """)


def test_more_heads_than_the_merge_counts_are_refused(runtime):  # noqa: F811
    """The merge finds a state by a 32-bit byte address (2^23 columns of 512 bytes) and its request by quotients below 2^20."""
    go(runtime, """
        for n, hq, hkv in ((1024, 1024, 1024), (1024, 8192, 512), (1024, 4096, 256), (600, 2048, 2048), (512, 8192, 512)):
            assert refused(shared, make_pool(hq=hq, hkv=hkv), n=n), (n, hq, hkv)
        for n, hq, hkv in ((1024, 1023, 1023), (1024, 4000, 250), (512, 2047, 2047), (500, 8000, 500)):
            shared(make_pool(hq=hq, hkv=hkv), n=n)
    """)
