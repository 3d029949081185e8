"""Refusals and launches of the calls on a batch's rows around the attention, on the stand-in HIP runtime (no GPU;
tests/test_host_dispatch.py): what a call refuses launches nothing, what it takes launches what is written here."""
import textwrap

import pytest

from tests.test_host_dispatch import CXX, run, runtime  # noqa: F401

pytestmark = pytest.mark.skipif(CXX is None, reason="needs g++")

CALLS = """
    SLOT, RES, WB, WN, GATE, ITEMS, ORDER, SCRATCH, TOKENS = ((i + 30) << 32 for i in range(9))


    def norm(p, n=5, how=None, block=Q, bs=1024, res=RES, rs=1024, slot=None, out=OUT, x=K, **kw):
        args = dict(width=1024, next_weight=WN)
        args.update(kw)
        p.odma_add_norm(n, B.make_add_norm(**args) if how is None else how, block, bs, res, rs, slot, out, x, 0)

    def group(p, n=8, adapter=LENS, n_adapters=4, start=OFFS, max_rows=640, order=ORDER, max_items=14, items=ITEMS):
        p.odma_group_adapters(n, adapter, n_adapters, start, max_rows, order, max_items, items, 0)

    def make(down=WB, up=WN, n_adapters=4, rank=16, width=512, part_cols=(64, 32), **kw):
        return B.make_adapters(down=down, up=up, n_adapters=n_adapters, rank=rank, width=width, part_cols=part_cols, **kw)

    def adapt(p, n=100, ad=None, max_items=6, items=ITEMS, order=ORDER, x=Q, xs=512, base=K, bs=96, y=V, ys=96, scratch=SCRATCH, size=1 << 40):
        ad = make() if ad is None else ad
        rc = B.lib.odma_adapt_rows(p._h, n, ad, max_items, items, order, x, xs, base, bs, y, ys, scratch, size, None)
        if rc:
            raise B.OdmaError(rc, B.odma_last_error())

    def score(p, n=5, logits=Q, stride=32000, dtype=B.BF16, vocab=32000, scale=1.0, tokens=TOKENS, slot=None, top=5, lp=K, rank=V, ent=WS, ids=NEW,
              lps=OUT, scratch=SCRATCH, size=1 << 40):
        rc = B.lib.odma_score_tokens(p._h, n, logits, stride, dtype, vocab, scale, tokens, slot, top, lp, rank, ent, ids, lps, scratch, size, None)
        if rc:
            raise B.OdmaError(rc, B.odma_last_error())

    def refused(call, *a, **kw):
        at = hip.fake_launches()
        try:
            call(*a, **kw)
        except B.OdmaError as e:
            assert e.code == B.INVALID_ARG, e
            assert hip.fake_launches() == at
            return True
        return False

    def bare():
        cfg, keep = B.make_config(n_layers=1, n_q_heads=4, n_kv_heads=2, head_dim=64, kv_dtype=B.BF16, out_dtype=B.BF16, main_tokens=64,
                                  safety_tokens=64, large_cap=64, boundaries=(64,), quantiles=((1, 2),), max_requests=8)
        return B.Pool(cfg, keep)                                 # allocator only
"""


def go(runtime, code):  # noqa: F811
    run(runtime, textwrap.dedent(CALLS) + textwrap.dedent(code))


def test_add_norm(runtime):  # noqa: F811
    go(runtime, """
        p, f = make_pool(), make_pool(kv_dtype=B.F32)
        nan, inf = float("nan"), float("inf")
        for bad in (dict(n=-1), dict(n=(1 << 22) + 1), dict(res=None), dict(out=None, x=None, next_weight=None), dict(width=0), dict(width=-8),
                    dict(width=1020), dict(width=32776), dict(residual_dtype=B.FP8), dict(residual_dtype=7), dict(x=None), dict(next_weight=None), dict(x=Q, bs=2048),
                    dict(block=None, block_weight=WB), dict(block=None, gate=GATE), dict(gate=GATE, gate_kind=B.GATE_NONE),
                    dict(gate_kind=B.GATE_VALUE), dict(gate=GATE, gate_kind=3), dict(gate=GATE, gate_kind=-1), dict(eps=-1e-6), dict(eps=nan),
                    dict(eps=inf), dict(residual_scale=inf), dict(block_scale=nan), dict(block=Q + 8), dict(res=RES + 4), dict(out=OUT + 8),
                    dict(x=K + 2), dict(gate=GATE + 8), dict(block_weight=WB + 8), dict(next_weight=WN + 4), dict(bs=1028), dict(bs=-1024),
                    dict(rs=1028), dict(rs=-8), dict(gate=GATE, gate_stride=4), dict(gate=GATE, gate_stride=-8), dict(rs=1016), dict(rs=0)):
            assert refused(norm, p, **bad), bad
        assert refused(norm, f) and refused(norm, f, residual_dtype=B.BF16)    # (rows in fp32: the residual too)
        assert refused(norm, f, residual_dtype=B.F32, bs=1026) and refused(norm, bare())
        assert B.lib.odma_add_norm(p._h, 1, None, Q, 0, RES, 0, None, OUT, K, None) == B.INVALID_ARG
        assert launched(lambda: norm(p, n=0)) == []
        # a row for all; rows that stand apart; one residual for all, not kept
        norm(p, rs=0, n=1), norm(p, bs=0), norm(p, bs=4096, rs=2048, gate=GATE, gate_stride=0), norm(p, rs=0, out=None)
        norm(p, residual_dtype=B.F32, rs=1028), norm(f, residual_dtype=B.F32, bs=1028, rs=1028), norm(p, block=None, out=None)
        norm(make_pool(kv_dtype=B.FP8), slot=SLOT), norm(p, x=Q)
        # a wave for every 512 channels, rows of up to four waves side by side; with many rows fewer waves at some widths
        for n, width, wg in ((1, 512, 1), (5, 512, 2), (5, 1024, 3), (5, 2048, 5), (5, 4096, 5), (5, 32768, 5), (1023, 2048, 1023), (1024, 512, 256),
                             (16383, 1024, 8192), (16384, 1024, 4096), (1025, 2048, 1025), (49151, 3584, 49151), (49152, 3584, 24576), (1023, 8192, 1023),
                             (1025, 8192, 1025), (1025, 32768, 1025), (1 << 22, 32768, 1 << 22)):
            one = launched(lambda: norm(p, n=n, width=width, bs=width, rs=width))
            assert len(one) == 1 and "add_norm_kernel" in one[0][0] and one[0][1] == (wg, 1, 1), (n, width, one)
        hip.fake_fail_launch(0)
        assert fails(lambda: norm(p))
    """)


def test_group_adapters(runtime):  # noqa: F811
    go(runtime, """
        p = make_pool(max_requests=3000)
        for bad in (dict(n=-1), dict(n=3001), dict(adapter=None), dict(n_adapters=0), dict(n_adapters=65537), dict(max_rows=-1),
                    dict(max_rows=(1 << 27) + 1, max_items=1 << 30), dict(order=None), dict(items=None), dict(items=ITEMS + 8), dict(max_items=13)):
            assert refused(group, p, **bad), bad
        assert refused(group, bare())
        group(p, max_rows=0, order=None, max_items=4)
        group(p, n=2, max_items=12)                               # (two requests have two adapters at most)
        one = launched(lambda: group(p, n=0, adapter=None, max_items=10))
        assert len(one) == 1 and one[0][1] == (1, 1, 1)           # empty lists are written too
        assert launched(lambda: group(p, start=None))[0][1:] == ((8, 1, 1), 4)
        assert launched(lambda: group(p, n_adapters=65536, max_items=18))[0][2] == 8192
        # long requests are dealt out, many requests share work-groups; up to 1024 work-groups
        assert launched(lambda: group(p, max_rows=1 << 20, max_items=1 << 15))[0][1] == (8, 128, 1)
        assert launched(lambda: group(p, n=3000, n_adapters=65536, max_items=4000))[0][1] == (1000, 1, 1)
        hip.fake_fail_launch(0)
        assert fails(lambda: group(p))
    """)


def test_adapt_rows(runtime):  # noqa: F811
    go(runtime, """
        p, f = make_pool(), make_pool(kv_dtype=B.F32)
        for bad in (dict(n=-1), dict(n=(1 << 27) + 1), dict(items=None), dict(order=None), dict(x=None), dict(base=None), dict(y=None),
                    dict(scratch=None), dict(scratch=SCRATCH + 16), dict(size=0), dict(items=ITEMS + 4), dict(max_items=-1), dict(x=Q + 2),
                    dict(base=K + 8), dict(y=V + 8), dict(xs=516), dict(bs=100), dict(ys=100), dict(xs=-512), dict(bs=-96), dict(ys=88),
                    dict(y=K, ys=104), dict(max_items=1 << 23)):
            assert refused(adapt, p, **bad), bad
        for bad in (dict(down=None), dict(up=None), dict(down=WB + 8), dict(up=WN + 2), dict(n_adapters=0), dict(n_adapters=65537), dict(rank=0),
                    dict(rank=12), dict(rank=264), dict(width=0), dict(width=508), dict(width=32776), dict(part_cols=(64, 24)), dict(part_cols=(0, 32)),
                    dict(part_cols=(64, -32))):
            ad = make(**bad)
            assert refused(adapt, p, ad=ad), bad
            assert refused(p.odma_adapt_scratch_bytes, ad, 6), bad
        for cols in ((), (16,) * 5):
            try:
                make(part_cols=cols)
                assert False
            except ValueError:
                pass
        for n_parts in (0, 5):
            ad = make()
            ad.n_parts = n_parts
            assert refused(adapt, p, ad=ad)
        ad = make()
        ad.part_start[0] = 16
        assert refused(adapt, p, ad=ad)
        assert refused(adapt, bare()) and refused(p.odma_adapt_scratch_bytes, None, 6) and B.lib.odma_adapt_scratch_bytes(None, make(), 6) == 0
        assert launched(lambda: adapt(p, n=0)) == [] and launched(lambda: adapt(p, max_items=0)) == []
        assert p.odma_adapt_scratch_bytes(make(), 0) > 0
        size = p.odma_adapt_scratch_bytes(make(), 6)
        adapt(p, size=size)
        assert refused(adapt, p, size=size - 1)
        adapt(p, y=K, ys=96), adapt(f, xs=516, bs=100, ys=100), adapt(p, xs=0, bs=0)
        two = launched(lambda: adapt(p, ys=256, ad=make(rank=256, part_cols=(64, 64, 64, 64), width=32768)))
        assert ["down" in two[0][0], "up" in two[1][0]] == [True, True] and len(two) == 2 and two[1][2] == 32768
        # few rows take one launch, by the matrix instructions of a work-group and the rounds of them
        for pool, n, rank, width, few in ((p, 1, 16, 3584, True), (p, 8192, 16, 512, True), (p, 8193, 16, 512, False), (p, 1, 32, 3584, True), (p, 1, 64, 3584, False),
                                          (p, 100, 64, 3584, True), (p, 100, 64, 8192, False), (p, 8192, 64, 512, True), (p, 8192, 64, 3584, False),
                                          (p, 200, 72, 512, False), (f, 1, 16, 3584, False), (f, 1, 16, 1024, True), (f, 200, 64, 3584, False), (f, 800, 64, 3584, True),
                                          (f, 1, 8, 1024, True), (f, 8192, 64, 8192, False), (f, 128, 72, 512, False)):
            got = launched(lambda: adapt(pool, n=n, ad=make(rank=rank, width=width), xs=width))
            assert len(got) == (1 if few else 2) and ("few" in got[0][0]) == few, (n, rank, width, got)
        assert len(launched(lambda: adapt(p, max_items=1025))) == 2
        assert launched(lambda: adapt(p, n=100))[0][1] == (2 * 16, 1, 1)       # 6 + 6 runs of 16 rows, in eights; two parts of a chunk of columns each
        # long calls pass rows by the caches, where their lines are whole; groups of ranks take items in 32s
        assert "Lb1E" in launched(lambda: adapt(p, n=100000, max_items=1600, ys=4608, bs=4608, ad=make(part_cols=(3584, 512, 512))))[1][0]
        for part_cols, ys, rank, stream, first in (((3584, 512, 512), 4608, 16, True, 1590), ((3584, 512, 512), 4616, 16, False, 1590),
                                                   ((3600, 496, 512), 4608, 16, False, 1590), ((3584, 512, 512), 4672, 64, True, 1600 * 3)):
            got = launched(lambda: adapt(p, n=100000, max_items=1590, ys=ys, bs=4608, ad=make(part_cols=part_cols, rank=rank)))
            assert ("Lb1E" in got[1][0]) == stream and got[0][1][0] == first, got
        for at, kw in ((0, {}), (0, dict(n=9000)), (1, dict(n=9000))):
            hip.fake_fail_launch(at)
            assert fails(lambda: adapt(p, **kw))
    """)


def test_score_tokens(runtime):  # noqa: F811
    go(runtime, """
        p = make_pool()
        nan, inf = float("nan"), float("inf")
        for bad in (dict(n=-1), dict(n=(1 << 22) + 1), dict(logits=None), dict(dtype=B.FP8), dict(dtype=-1), dict(vocab=0), dict(vocab=-4),
                    dict(vocab=(1 << 24) + 1, stride=1 << 25), dict(stride=31999), dict(stride=-32000), dict(logits=Q + 1),
                    dict(logits=Q + 2, dtype=B.F32), dict(scale=0.0), dict(scale=-1.0), dict(scale=nan), dict(scale=inf), dict(scale=1e-8),
                    dict(scale=1e8), dict(tokens=None), dict(tokens=None, lp=None), dict(tokens=None, rank=None), dict(top=-1), dict(top=65),
                    dict(vocab=4), dict(top=0), dict(top=0, ids=None), dict(top=0, lps=None), dict(ids=None, lps=None),
                    dict(top=0, ids=None, lps=None, lp=None, rank=None, ent=None), dict(scratch=None), dict(scratch=SCRATCH + 128), dict(size=0)):
            assert refused(score, p, **bad), bad
        assert refused(score, bare()) and B.lib.odma_score_scratch_bytes(None, 5, 100, 5) == 0
        for bad in ((-1, 100, 5), ((1 << 22) + 1, 100, 5), (5, 0, 0), (5, (1 << 24) + 1, 5), (5, 100, 65), (5, 4, 5), (5, 100, -1)):
            assert refused(p.odma_score_scratch_bytes, *bad), bad
        assert launched(lambda: score(p, n=0)) == []
        size = p.odma_score_scratch_bytes(5, 32000, 5)
        score(p, size=size)
        assert refused(score, p, size=size - 1)
        # results that nobody asks for
        score(p, tokens=None, lp=None, rank=None), score(p, top=0, ids=None, lps=None), score(p, ids=None), score(p, lps=None, ent=None)
        score(p, n=1, stride=0), score(p, logits=Q + 2, stride=32001), score(p, logits=Q + 4, stride=32001, dtype=B.F32, scale=2.0 ** -24)
        # rows of up to 32 768 tokens are whole; longer ones of few rows are cut into parts of 2048 or more, 64 at most, which a second launch
        # joins.  Waves of a work-group: 4, of 16 to 256 rows (and of short rows up to there) 16, up to 512 rows 8
        for n, vocab, wg, waves in ((1, 5, 1, 16), (1, 32768, 1, 16), (1, 32769, 17, 4), (1, 1 << 24, 64, 4), (15, 128000, 945, 4), (16, 128000, 256, 16),
                                    (100, 128000, 200, 16), (256, 128000, 256, 16), (256, 300, 256, 16), (257, 300, 257, 8), (512, 128000, 512, 8),
                                    (513, 128000, 513, 4), (1 << 22, 5, 1 << 22, 4)):
            got = launched(lambda: score(p, n=n, vocab=vocab, stride=vocab))
            assert "score_kernel" in got[0][0] and f"Li{waves}E" in got[0][0] and got[0][1] == (wg, 1, 1), (n, vocab, got)
            assert len(got) == (2 if wg > n else 1) and (wg == n or (got[1][1] == (n, 1, 1) and "join" in got[1][0]))
        for at in (0, 1):
            hip.fake_fail_launch(at)
            assert fails(lambda: score(p, vocab=128000, stride=128000))
    """)
