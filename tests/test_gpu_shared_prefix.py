"""odma_decode_attention_shared against attention of every request by itself, in 64 bits.  Pools are filled with NaN patterns
first, so that a slot no request holds shows where it is read."""
import math

import numpy as np
import pytest
import torch

import workloads as wl
from oracle import attention as oa
from paper_2512_09427_amd import binding as B
from tests import harness as H
from tests.test_gpu_parity import small_workload

pytestmark = pytest.mark.gpu


class Batch:
    """Requests with own rows behind shared ones: lengths count both.  groups: (first request, behind the last, prefix length)."""

    def __init__(self, lengths, groups, *, kvd="bf16", hq=28, hkv=4, d=128, out=B.F32, paged=False, seed=0, scale=1.0, edit=None):
        self.n, self.kvd, self.paged, self.hq, self.hkv, self.d, self.out = len(lengths), kvd, paged, hq, hkv, d, out
        rng = np.random.default_rng(seed)
        self.lengths = np.asarray(lengths, np.int64)
        self.start = np.array([g[0] for g in groups] + [groups[-1][1]], np.int32)
        assert all(a[1] == b[0] for a, b in zip(groups, groups[1:]))
        self.plen = np.array([g[2] for g in groups], np.int32)
        self.group = np.full(self.n, -1)
        for p, (a, b, _) in enumerate(groups):
            self.group[a:b] = p
        whole = np.append(np.maximum(self.plen, 0) // 16 * 16, 0)
        self.shared = whole[self.group]
        own = np.maximum(self.lengths - self.shared, 0)
        # every request and every prefix is a request of the pool
        rows = np.concatenate([own, np.maximum(self.plen, 0)])
        cap = int(max(rows.max(), 1) + 15) // 16 * 16
        w = small_workload(rows, kv_dtype=kvd, hq=hq, hkv=hkv, d=d, bounds=(cap,), large_cap=cap,
                           main=int(((rows + 15) // 16 * 16).sum()) + 16 * len(rows) + 16, safety=cap)
        self.w, self.dp = w, H.make_pool(w, out_dtype=out, max_requests=len(rows), quantiles=((1, 2),))
        value = lambda shape, size: wl.draw_values(rng, shape, size, "bf16" if kvd == "bf16" else kvd)[0]  # noqa: E731
        self.kv = [(value((c, hkv, d), scale), value((c, hkv, d), 1.0)) for c in rows]
        self.q = wl.draw_values(rng, (self.n, hq, d), 1.0, "bf16")[0]
        if edit:
            edit(self)
        blocks = (rows + 15) // 16
        base = (np.cumsum(blocks) - blocks + np.arange(len(rows))) * 16          # a block nobody has between slabs
        self.place = rng.permutation(w.main_tokens // 16) if paged else None
        if paged:
            width = max(int(blocks.max()), 1)
            mine = np.array([[self.place[b // 16 + min(j, max(c - 1, 0))] for j in range(width)] for b, c in zip(base, blocks)], np.int32)
            H.fill(self.dp, 0, self.kv, block_table=mine)
            stride = int((max(self.lengths.max(), 1) + 15) // 16) + 1
            # entries behind a request's last block name a block full of NaN
            table = np.full((self.n, stride), self.place[-1], np.int32)
            for r in range(self.n):
                s = self.shared[r] // 16
                for j in range(int(self.lengths[r] + 15) // 16):
                    table[r, j] = mine[self.n + self.group[r], j] if j < s else mine[r, j - s]
            self.table, self.offsets, self.poff = table, None, None
        else:
            H.fill(self.dp, 0, self.kv, offsets=base)
            self.table, self.offsets, self.poff = None, base[:self.n].astype(np.int64), base[self.n:].astype(np.int64)

    def rows_of(self, r):
        """The K and V rows that request r attends to."""
        n, s = int(self.lengths[r]), int(self.shared[r])
        pre = self.kv[self.n + self.group[r]] if s else self.kv[r]
        return tuple(np.concatenate([pre[i][:min(s, n)], self.kv[r][i][:max(n - s, 0)]]) for i in range(2))

    def tensors(self):
        put = lambda a, t: None if a is None else H.to_dev(np.asarray(a, t))  # noqa: E731
        res = torch.full((self.n, self.hq, self.d), -1 if self.out == B.BF16 else float("nan"), dtype=self.dp.out_torch_dtype, device=H.DEV)
        return dict(q=H.to_dev(self.q), start=put(self.start, np.int32), poff=put(self.poff, np.int64), plen=put(self.plen, np.int32),
                    off=put(self.offsets, np.int64), lens=put(self.lengths, np.int32), bt=put(self.table, np.int32), out=res)

    def call(self, t, prefixes=None, stream=None):
        self.dp.pool.odma_decode_attention_shared(0, self.n, t["q"], len(self.plen) if prefixes is None else prefixes, t["start"], t["poff"],
                                                  t["plen"], t["off"], t["lens"], t["bt"], 0 if t["bt"] is None else t["bt"].shape[1],
                                                  t["out"], stream)
        return t["out"]

    def values(self, out):
        torch.cuda.synchronize()
        res = out.cpu().numpy()
        return wl.bf16_bits_to_f32(res.view(np.uint16)) if self.out == B.BF16 else res

    def reference(self):
        """The result, and sum p |v|, of which every rounding of a weight is a part."""
        sm = (wl.FP8_SCALE if self.kvd == "fp8" else 1.0) / math.sqrt(self.d)
        unit = wl.FP8_SCALE if self.kvd == "fp8" else 1.0
        ref, size = np.zeros((self.n, self.hq, self.d)), np.zeros((self.n, self.hq, self.d))
        absolute = {"bf16": 0x7fff, "fp8": 0x7f}[self.kvd]
        for r in range(self.n):
            k, v = self.rows_of(r)
            if len(k):
                ref[r] = oa.attend_one(self.q[r], k, v, sm) * unit
                size[r] = oa.attend_one(self.q[r], k, (v & absolute).astype(v.dtype), sm) * unit
        return ref, size

    def check(self, got, ref, size, scores=4.0):
        # A weight is off by the fp32 sum of its score (128 terms of size up to |score|: 2^-20 of it) and by the exponential (2^-22).
        # fp32 results keep all bits of a weight; results in bf16 let the weights of shared tokens be one bf16 number (2^-8), of own
        # ones two (2^-16).  States are joined by factors that are off by an exponential (2^-22) each.
        weight = 2.0 ** -21 + scores * 2.0 ** -19 + (2.0 ** -8 + 2.0 ** -16 if self.out == B.BF16 else 0.0)
        bound = weight * size + (2.0 ** -8 if self.out == B.BF16 else 2.0 ** -23) * np.abs(ref) + 1e-30
        err = np.abs(got.astype(np.float64) - ref)
        assert np.isfinite(got).all() and (err <= bound).all(), (err / bound).max()
        assert (got[self.lengths == 0] == 0).all()

    def run(self, **kw):
        got = self.values(self.call(self.tensors()))
        self.check(got, *self.reference(), **kw)
        return got


FORMATS = [("bf16", 128), ("bf16", 64), ("fp8", 128)]
# lengths, groups (first, behind the last, prefix length)
CASES = {
    "one request": ([40], [(0, 1, 16)]),
    "nothing of its own": ([16, 48], [(0, 1, 16), (1, 2, 48)]),
    "ragged": ([1000, 993, 992, 1500, 1024, 0, 2300, 1001], [(0, 8, 1000)]),
    "odd numbers of tiles": ([60, 49, 90, 17, 16, 81, 80, 100], [(0, 3, 48), (3, 5, 16), (5, 8, 80)]),
    "shorter than the shared part": ([10, 200, 159, 160, 161, 0, 1, 400], [(0, 8, 160)]),
    "all shorter": ([10, 100, 31], [(0, 3, 160)]),
    "all empty": ([0, 0, 0], [(0, 3, 160)]),
    "an empty place first": ([0, 0, 300, 180, 0, 250], [(0, 3, 170), (3, 6, 100)]),
    "no whole block, none, less than none": ([50, 20, 70, 1, 33], [(0, 2, 15), (2, 3, 0), (3, 5, -7)]),
    "groups and places outside": ([30, 0, 500, 700, 650, 5, 90, 90], [(1, 4, 400), (4, 4, 64), (4, 6, 200)]),
    "a prefix of its own each": ([100, 130, 260, 70], [(0, 1, 90), (1, 2, 128), (2, 3, 17), (3, 4, 64)]),
}


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("kvd,d", FORMATS)
@pytest.mark.parametrize("name", list(CASES))
def test_small_batches(name, kvd, d, paged):
    lengths, groups = CASES[name]
    Batch(lengths, groups, kvd=kvd, d=d, paged=paged, hq=7, hkv=1, seed=len(name)).run()
    Batch(lengths, groups, kvd=kvd, d=d, paged=paged, hq=6, hkv=3, seed=len(name), out=B.BF16).run()


@pytest.mark.parametrize("hq,hkv", [(1, 1), (16, 1), (32, 2), (8, 8), (28, 4), (10, 2)])
@pytest.mark.parametrize("kvd,d", FORMATS)
def test_head_layouts(kvd, d, hq, hkv):
    """Columns of one request to sixteen heads of a group; blocks of 128 columns that end inside a request."""
    rng = np.random.default_rng(hq)
    lengths = 320 + rng.integers(0, 200, 21)
    Batch(lengths, [(0, 9, 325), (9, 21, 100)], kvd=kvd, d=d, hq=hq, hkv=hkv, seed=hq).run()


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("out", [B.F32, B.BF16])
@pytest.mark.parametrize("kvd,d", FORMATS)
def test_long_prefixes_are_cut(kvd, d, out, paged):
    """A prefix of thousands of tokens for few requests, beside a long request: both lines are cut many times."""
    Batch([9000, 9500, 16000, 9100, 8999, 7000], [(0, 5, 9003)], kvd=kvd, d=d, hq=8, hkv=2, out=out, paged=paged).run()


@pytest.mark.parametrize("out", [B.F32, B.BF16])
@pytest.mark.parametrize("kvd,d", FORMATS)
@pytest.mark.parametrize("hq,hkv,lengths,prefix", [(1, 1, [30000], 9000), (1, 1, [20003, 4, 0], 20000), (5, 1, [20, 30001], 30623), (28, 4, [9000, 9500, 16000, 9100, 8999, 7000], 9003)])
def test_many_pieces_of_few_heads(hq, hkv, lengths, prefix, kvd, d, out):
    """Prefixes and own tokens cut into hundreds of pieces, for as few heads as four waves join each, and for more."""
    Batch(lengths, [(0, len(lengths), prefix)], kvd=kvd, d=d, hq=hq, hkv=hkv, out=out, seed=hq).run()


@pytest.mark.parametrize("n,hq,hkv,prefixes", [(300, 28, 4, 3), (1024, 4, 2, 1), (1024, 2, 1, 1024), (777, 16, 1, 50), (1000, 1, 1, 2)])
def test_many_requests(n, hq, hkv, prefixes):
    rng = np.random.default_rng(n)
    cuts = np.sort(rng.integers(0, n + 1, prefixes + 1)) if prefixes < n else np.arange(n + 1)
    plens = rng.integers(1, 300, prefixes) if prefixes > 1 else [700]
    groups = [(int(a), int(b), int(p)) for a, b, p in zip(cuts, cuts[1:], plens)]
    lengths = rng.integers(0, 400, n)
    for a, b, p in groups:
        lengths[a:b] += p * (rng.random(b - a) < 0.8)
    Batch(lengths, groups, hq=hq, hkv=hkv, seed=n).run()


@pytest.mark.parametrize("paged", [False, True])
def test_scores_that_grow_and_fall(paged):
    """References that have to move, and pieces whose largest scores lie far from one another."""
    def edit(b):
        for r, (k, v) in enumerate(b.kv):
            t = np.arange(len(k))
            steps = np.where(t < len(k) // 2, 300.0, -300.0) * np.sin(t / 40.0) * (1 + r % 3) / 2
            k[:, :, 0] = wl.f32_to_bf16_bits(steps.astype(np.float32))[:, None]
        b.q[:, :, 0] = wl.f32_to_bf16_bits(np.float32(2.0))

    # (scores up to 600 / 11.3 = 53)
    Batch([3000, 2500, 2111, 5000, 2000], [(0, 4, 2050)], hq=8, hkv=2, paged=paged, edit=edit).run(scores=64.0)


@pytest.mark.parametrize("out", [B.F32, B.BF16])
def test_tokens_switched_off_and_infinite_values(out):
    """Tokens that score -inf in the prefix, in the own part, in whole pieces; V infinite in some channels of one token."""
    off = wl.f32_to_bf16_bits(np.float32(-np.inf))

    def edit(b):
        for k, _ in b.kv:
            k[:, :, 0] = 0
        b.q[:, :, 0] = wl.f32_to_bf16_bits(np.float32(1.0))
        prefix = b.kv[b.n][0]
        prefix[:700, :, 0] = off
        prefix[1000:1040, :, 0] = off
        b.kv[1][0][:, :, 0] = off                                        # a request whose own tokens are all off
        b.kv[2][0][:33, :, 0] = off
        b.kv[3][1][5, :, 3::7] = wl.f32_to_bf16_bits(np.float32(np.inf))
        b.kv[b.n][1][900, :, 4::9] = wl.f32_to_bf16_bits(np.float32(-np.inf))

    b = Batch([2000, 2040, 2100, 2500, 1990], [(0, 5, 1980)], hq=8, hkv=2, out=out, edit=edit)
    got = b.values(b.call(b.tensors()))
    with np.errstate(invalid="ignore"):
        ref, size = b.reference()
    # (channels 31 and 94 of request 3 sum infinities of both signs: not a number)
    inf = ~np.isfinite(ref)
    assert np.isinf(ref).any() and np.isnan(ref).sum() == np.isnan(ref[3][:, [31, 94]]).sum() == 16
    np.testing.assert_array_equal(got[inf], ref[inf])
    b.check(np.where(inf, 0, got), np.where(inf, 0, ref), np.where(inf, 0, size))


def test_a_request_without_a_finite_score_touches_no_other():
    off = wl.f32_to_bf16_bits(np.float32(-np.inf))

    def edit(b):
        for r, (k, _) in enumerate(b.kv):
            k[:, :, 0] = off if r in (1, b.n) else 0
        b.q[:, :, 0] = wl.f32_to_bf16_bits(np.float32(1.0))

    b = Batch([100, 120, 0, 300], [(0, 3, 64)], hq=4, hkv=2, edit=edit)
    got = b.values(b.call(b.tensors()))
    assert np.isnan(got[1]).all()
    ref, size = b.reference()
    for a in (got, ref, size):
        a[1] = 0
    b.check(got, ref, size)


def test_nan_in_one_request_touches_no_other():
    def edit(b):
        b.q[2] = 0x7fff
        b.kv[3][1][7] = 0x7fff

    b = Batch([400, 380, 400, 500, 450, 420], [(0, 6, 370)], hq=14, hkv=2, edit=edit)
    clean = Batch([400, 380, 400, 500, 450, 420], [(0, 6, 370)], hq=14, hkv=2)
    got, want = (x.values(x.call(x.tensors())) for x in (b, clean))
    assert np.isnan(got[[2, 3]]).all()
    keep = [0, 1, 4, 5]
    np.testing.assert_array_equal(got[keep], want[keep])


@pytest.mark.parametrize("kvd,d", FORMATS)
@pytest.mark.parametrize("paged", [False, True])
def test_without_prefixes_it_is_a_decode_call(kvd, d, paged):
    b = Batch([100, 1, 0, 777, 33], [(0, 5, 0)], kvd=kvd, d=d, paged=paged, hq=8, hkv=2)
    got = b.values(b.call(b.tensors(), prefixes=0))
    where = dict(block_table=b.table) if paged else dict(offsets=b.offsets)
    np.testing.assert_array_equal(got, H.decode(b.dp, 0, b.q, b.lengths, **where))


def test_a_plan_survives_and_calls_repeat_bit_for_bit():
    """A workspace full of anything; decode calls that reuse their plan around the call; the same result every time."""
    b = Batch([1500, 1400, 2222, 1333, 1600], [(0, 5, 1300)], hq=28, hkv=4)
    b.dp.workspace.fill_(255)
    t = b.tensors()
    want = b.call(t).clone()
    own = np.maximum(b.lengths - b.shared, 0)
    decoded = H.decode(b.dp, 0, b.q, own, offsets=b.offsets)
    for _ in range(3):
        t["out"].fill_(float("nan"))
        assert torch.equal(b.call(t), want)
        np.testing.assert_array_equal(H.decode(b.dp, 0, b.q, own, offsets=b.offsets, flags=B.REUSE_PLAN), decoded)
    b.check(b.values(want), *b.reference())


@pytest.mark.parametrize("paged", [False, True])
def test_captured_replayed_and_on_another_stream(paged):
    """One capture serves lengths that change between its replays; the program decodes eagerly between them."""
    b = Batch([900, 0, 1200, 880, 1000, 17], [(0, 5, 871)], hq=8, hkv=2, paged=paged, out=B.F32)
    t = b.tensors()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        b.call(t)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.call(t)
    full = b.lengths.copy()
    for shrink in (0, 3, 16, 880, 100000):
        b.lengths = np.maximum(full - shrink, 0)
        t["lens"].copy_(H.to_dev(b.lengths.astype(np.int32)))
        t["out"].fill_(float("nan"))
        graph.replay()
        got = b.values(t["out"])
        b.check(got, *b.reference())
        np.testing.assert_array_equal(b.values(b.call(t)), got)


def test_prefix_of_its_pool_alone_is_read():
    """Layers: the call reads the layer that it names."""
    w = small_workload([64, 64, 64], hq=4, hkv=2, bounds=(64,), large_cap=64, main=512, safety=64)
    dp = H.make_pool(w, out_dtype=B.F32, n_layers=2, quantiles=((1, 2),))
    rng = np.random.default_rng(0)
    kv = [[tuple(wl.draw_values(rng, (64, 2, 128), 1.0, "bf16")[0] for _ in range(2)) for _ in range(3)] for _ in range(2)]
    for layer in range(2):
        H.fill(dp, layer, kv[layer], offsets=np.array([0, 64, 128]))
    q = wl.draw_values(rng, (2, 4, 128), 1.0, "bf16")[0]
    dev = lambda a, t: H.to_dev(np.asarray(a, t))  # noqa: E731
    for layer in range(2):
        out = torch.empty(2, 4, 128, device=H.DEV)
        dp.pool.odma_decode_attention_shared(layer, 2, H.to_dev(q), 1, dev([0, 2], np.int32), dev([128], np.int64), dev([64], np.int32),
                                             dev([0, 64], np.int64), dev([128, 100], np.int32), None, 0, out)
        torch.cuda.synchronize()
        for r, own in enumerate((64, 36)):
            k, v = (np.concatenate([kv[layer][2][i], kv[layer][r][i][:own]]) for i in range(2))
            np.testing.assert_allclose(out[r].cpu().numpy(), oa.attend_one(q[r], k, v, 1 / math.sqrt(128)), atol=2.0 ** -13)


def number(kvd, x):
    """A number as K and V hold it."""
    return wl.f32_to_e4m3_bits(np.array([x], np.float32))[0] if kvd == "fp8" else wl.f32_to_bf16_bits(np.float32(x))


@pytest.mark.parametrize("empty", [False, True])
@pytest.mark.parametrize("hq", [16, 8])
@pytest.mark.parametrize("out", [B.F32, B.BF16])
@pytest.mark.parametrize("kvd,d", FORMATS)
def test_a_nan_query_leaves_its_neighbours_references_moving(kvd, d, out, hq, empty):
    """Scores that climb by more exponent units than a weight has, behind 32 tokens of low ones, beside a query that is NaN: of a live
    request, or of an empty place, whose queries nobody has to fill.  The columns of one head of requests 0 and 1 (of requests 0 and 2
    with eight heads) are sixteen apart."""
    def edit(b):
        # pairs of tiles score -7 q and 7 q in turn (q / sqrt(d) x 7: 53 to 76 either way)
        high, low = (number(kvd, x / (wl.FP8_SCALE if kvd == "fp8" else 1.0)) for x in (7.0, -7.0))
        for k, _ in b.kv:
            k[:, :, 0] = np.where(np.arange(len(k)) // 32 % 2, high, low)[:, None]
        b.q[:, :, 0] = wl.f32_to_bf16_bits(np.float32(87.0))
        b.q[0] = 0x7fff

    b = Batch([0 if empty else 530, 540, 520, 533], [(0, 4, 512)], kvd=kvd, d=d, hq=hq, hkv=1, out=out, seed=d, edit=edit)
    got = b.values(b.call(b.tensors()))
    assert (got[0] == 0).all() if empty else np.isnan(got[0]).all()
    b.q[0] = 0
    ref, size = b.reference()
    for a in (got, ref, size):
        a[0] = 0
    b.check(got, ref, size, scores=7 * 87 / math.sqrt(d) + 6)


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("low", [3e3, 1e5, 1e9])
@pytest.mark.parametrize("out", [B.F32, B.BF16])
@pytest.mark.parametrize("kvd,d", FORMATS)
def test_tokens_switched_off_by_large_finite_scores(kvd, d, out, low, paged):
    """Tokens far below the others, but finite: the first ones of a prefix, of a piece of it and of a request's own, a stretch inside,
    a whole prefix.  The scores of those that count keep all their bits."""
    one = number(kvd, -1.0 / (wl.FP8_SCALE if kvd == "fp8" else 1.0))

    def edit(b):
        for k, _ in b.kv:
            k[:, :, 0] = 0
        b.q[:, :, 0] = wl.f32_to_bf16_bits(np.float32(low))
        for tokens in (slice(0, 32), slice(128, 192), slice(330, 400), slice(512, 544), slice(640, 641)):
            b.kv[b.n][0][tokens, :, 0] = one
        b.kv[b.n + 1][0][:, :, 0] = one
        b.kv[0][0][:40, :, 0] = one
        b.kv[1][0][33:70, :, 0] = one

    Batch([868, 900, 769, 768, 160, 100], [(0, 4, 770), (4, 6, 96)], kvd=kvd, d=d, hq=8, hkv=2, out=out, paged=paged, seed=d, edit=edit).run()


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("low", [1e12, 1e30, 3e38])
@pytest.mark.parametrize("out", [B.F32, B.BF16])
@pytest.mark.parametrize("kvd,d", FORMATS)
def test_scores_whose_rounding_is_more_than_an_exponent_holds(kvd, d, out, low, paged):
    """Tokens switched off by scores near the lowest finite number, among others and alone (then all of them weigh the same)."""
    one = number(kvd, -1.0)

    def edit(b):
        for k, _ in b.kv:
            k[:, :, 0] = 0
        b.q[:, :, 0] = wl.f32_to_bf16_bits(np.float32(low))
        b.kv[b.n][0][:50, :, 0] = one
        b.kv[b.n + 1][0][:, :, 0] = one
        b.kv[0][0][:40, :, 0] = one
        b.kv[1][0][33:70, :, 0] = one
        b.kv[4][0][:, :, 0] = one
        b.q[4][:, 1:] = 0                                                # (all its scores are the same number)

    Batch([300, 370, 257, 170, 140], [(0, 3, 256), (3, 5, 96)], kvd=kvd, d=d, hq=8, hkv=2, out=out, paged=paged, seed=d, edit=edit).run()


@pytest.mark.parametrize("out", [B.F32, B.BF16])
@pytest.mark.parametrize("kvd,d", [f for f in FORMATS if f[0] == "bf16"])
def test_infinite_values_of_small_weights(kvd, d, out):
    """A token whose weight is 2^-80 to 2^-123 of the largest one's: its infinite V is an infinite result, of shared and of own tokens."""
    def edit(b):
        for k, _ in b.kv:
            k[:, :, 0] = 0
        b.q[:, :, 0] = wl.f32_to_bf16_bits(np.float32(1.0))
        # the others score 0 +- 1 in exponent units, the small ones 80, 81, .. less
        b.q[:, :, 1:] = wl.f32_to_bf16_bits(wl.bf16_bits_to_f32(b.q[:, :, 1:]) / 8)
        unit = math.sqrt(d) * math.log(2.0)
        for rows, at in ((b.kv[b.n], 200), (b.kv[1], 20)):
            for i in range(44):
                rows[0][at + i, :, 0] = wl.f32_to_bf16_bits(np.float32(-(80 + i) * unit))
                rows[1][at + i, :, i] = wl.f32_to_bf16_bits(np.float32(np.inf if i % 2 else -np.inf))

    b = Batch([600, 660, 601], [(0, 3, 520)], kvd=kvd, d=d, hq=4, hkv=2, out=out, seed=d, edit=edit)
    got = b.values(b.call(b.tensors()))
    with np.errstate(invalid="ignore"):
        ref, size = b.reference()
    inf = np.isinf(ref)
    assert not np.isnan(ref).any() and inf[:, :, :44].all() and not inf[:, :, 44:].any()
    np.testing.assert_array_equal(got[inf], ref[inf])
    b.check(np.where(inf, 0, got), np.where(inf, 0, ref), np.where(inf, 0, size))


@pytest.mark.parametrize("paged", [False, True])
def test_decode_calls_around_one_without_prefixes(paged):
    """A call without prefixes for other lengths between decode calls that ask for their earlier plan."""
    b = Batch([900, 40, 333, 1200], [(0, 4, 0)], hq=8, hkv=2, paged=paged)
    where = dict(block_table=b.table) if paged else dict(offsets=b.offsets)
    want = H.decode(b.dp, 0, b.q, b.lengths, **where)
    t = b.tensors()
    full, b.lengths = b.lengths, np.array([100, 40, 20, 640])
    t["lens"].copy_(H.to_dev(b.lengths.astype(np.int32)))
    b.check(b.values(b.call(t, prefixes=0)), *b.reference())
    for _ in range(2):
        np.testing.assert_array_equal(H.decode(b.dp, 0, b.q, full, flags=B.REUSE_PLAN, **where), want)


@pytest.mark.parametrize("out", [B.F32, B.BF16])
@pytest.mark.parametrize("kvd,d", FORMATS)
def test_what_an_empty_place_holds_changes_no_bit(kvd, d, out):
    """Queries of an empty place inside a group are whatever their memory held: zeros, large numbers, infinities, NaN."""
    b = Batch([700, 0, 715, 690, 0, 720], [(0, 6, 680)], kvd=kvd, d=d, hq=8, hkv=2, out=out, seed=d)
    want = b.run()
    held = [np.zeros_like(b.q[1])]
    for size in (3.0, 1e3, 1e20):
        held.append(wl.draw_values(np.random.default_rng(int(size) % 97), b.q[1].shape, size, "bf16")[0])
    held += [np.full_like(b.q[1], 0x7f80), np.full_like(b.q[1], 0x7fff)]
    for x in held:
        b.q[1] = b.q[4] = x
        np.testing.assert_array_equal(b.values(b.call(b.tensors())), want)
