"""odma_group_adapters against lists made on the host, and odma_adapt_rows against its formula: exactly, where inputs are whole numbers
and every sum is exact, and in 64 bits otherwise; both types, ranks, parts, ragged ranks, items of one row and of 64, batches that cut
the channels between work-groups and such that do not, strides, rows in no list, in place, streams and captured calls."""
import numpy as np
import pytest
import torch

from paper_2512_09427_amd import binding as B

DEV = "cuda"
pytestmark = pytest.mark.gpu
TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
ITEM = B.ADAPTER_ITEM_ROWS


def pool(typ="bf16", n=2048):
    kv = torch.zeros(2 * 80 * 32, dtype=TYPE[typ], device=DEV)
    t = B.F32 if typ == "f32" else B.BF16
    return B.Pool(*B.make_config(n_layers=1, n_q_heads=2, n_kv_heads=2, head_dim=32, kv_dtype=t, out_dtype=t, main_tokens=64, safety_tokens=16,
                                 large_cap=16, boundaries=(16,), quantiles=((1, 2),), max_requests=n, k_pool=kv, v_pool=kv.clone()))


def lists(adapter, rows, n_adapters, max_rows, max_items):
    start = np.cumsum(rows) - rows
    order, items = np.full(max_rows, -1), np.tile(np.array([B.ADAPTER_NONE, 0, 0, 0]), (max_items, 1))
    at, seen = 0, 0
    for a in sorted({int(x) for x, r in zip(adapter, rows) if 0 <= x < n_adapters and r}):
        first = at
        for r in np.flatnonzero(adapter == a):
            for j in range(rows[r]):
                if at < max_rows:
                    order[at] = start[r] + j
                at += 1
        for j in range(0, at - first, ITEM):
            if first + j < max_rows:
                items[first // ITEM + seen + j // ITEM] = a, first + j, min(ITEM, at - first - j, max_rows - first - j), 0
        seen += 1
    return order, items


def group(p, adapter, rows, n_adapters, *, max_rows=None, spare=0, start=True, stream=None):
    n, total = len(adapter), int(sum(rows))
    max_rows = total if max_rows is None else max_rows
    max_items = max_rows // ITEM + min(n, n_adapters) + spare
    order = torch.full((max_rows + 8,), 77, dtype=torch.int32, device=DEV)
    items = torch.full((max_items + 2, 4), 77, dtype=torch.int32, device=DEV)
    ad = torch.tensor(np.asarray(adapter), dtype=torch.int32, device=DEV)
    rs = torch.tensor(np.concatenate([[0], np.cumsum(rows)]), dtype=torch.int64, device=DEV) if start else None
    p.odma_group_adapters(n, ad if n else None, n_adapters, rs, max_rows, order, max_items, items, stream)
    torch.cuda.synchronize()
    assert (order[max_rows:] == 77).all() and (items[max_items:] == 77).all()
    return order[:max_rows], items[:max_items]


@pytest.mark.parametrize("n,n_adapters,most", [(1, 1, 1), (3, 5, 1), (64, 64, 1), (257, 7, 1), (1000, 65536, 1), (2000, 300, 1), (5, 2, 200), (40, 9, 70),
                                               (300, 33, 128), (1500, 4000, 9), (7, 65536, 5000)])
def test_lists(n, n_adapters, most):
    rng = np.random.default_rng(n + most)
    adapter = rng.integers(-1, n_adapters, n)
    adapter[rng.random(n) < 0.1] = rng.choice([-7, n_adapters, 2 ** 31 - 1, -2 ** 31])
    rows = np.ones(n, np.int64) if most == 1 else rng.integers(0, most + 1, n)
    p = pool()
    want = lists(adapter, rows, n_adapters, int(rows.sum()), int(rows.sum()) // ITEM + min(n, n_adapters) + 3)
    for start in ([True, False] if most == 1 else [True]):
        got = group(p, adapter, rows, n_adapters, spare=3, start=start)
        assert (got[0].cpu().numpy() == want[0]).all() and (got[1].cpu().numpy() == want[1]).all()


def test_lists_at_the_edges():
    p = pool()
    # nobody, nobody with an adapter, no rows
    for adapter, rows in (([], []), ([-1, 9, -1], [3, 4, 5]), ([1, 2], [0, 0])):
        order, items = group(p, np.array(adapter, np.int64), np.array(rows, np.int64), 9, max_rows=130)
        assert (order == -1).all() and (items == torch.tensor([-1, 0, 0, 0], device=DEV)).all()
    # all of one adapter, whole items and one row more; rows with no request in front of them are another's business
    for rows in ([64], [128], [129], [63, 1, 64], [1] * 65):
        ad = np.full(len(rows), 4)
        got, want = group(p, ad, np.array(rows), 5, spare=1), lists(ad, np.array(rows), 5, sum(rows), sum(rows) // ITEM + min(len(rows), 5) + 1)
        assert (got[0].cpu().numpy() == want[0]).all() and (got[1].cpu().numpy() == want[1]).all()
    # more rows than the lists hold: those past them do not exist
    rng = np.random.default_rng(1)
    ad, rows = rng.integers(0, 6, 50), rng.integers(0, 90, 50)
    for max_rows in (0, 1, 64, 500, int(rows.sum()) - 1, int(rows.sum()) + 200):
        got, want = group(p, ad, rows, 6, max_rows=max_rows), lists(ad, rows, 6, max_rows, max_rows // ITEM + 6)
        assert (got[0].cpu().numpy() == want[0]).all()
        assert (got[1].cpu().numpy() == want[1][:len(got[1])]).all()


class Case:
    """rows[r] rows of request r with adapter[r]; whole: inputs are whole numbers small enough for every sum to be exact."""

    def __init__(self, typ, adapter, rows, n_adapters, width, cols, rank, *, ranks=None, scale=True, whole=True, pads=(0, 0, 0), seed=0, spare=0):
        gen = torch.Generator().manual_seed(seed)
        self.typ, self.rank, self.width, self.cols, self.n_adapters, self.whole = typ, rank, width, cols, n_adapters, whole
        self.total, all_cols = int(sum(rows)), sum(cols)
        self.all_cols = all_cols

        def values(*shape, most=2, size=1.0):
            return torch.randint(-most, most + 1, shape, generator=gen).float() if whole else torch.randn(*shape, generator=gen) * size

        t = TYPE[typ]
        down, up = values(n_adapters, len(cols), rank, width, most=1, size=width ** -0.5), values(n_adapters, all_cols, rank, most=1)
        ranks_used = [rank] * n_adapters if ranks is None else [min(max((r + 7) // 8 * 8, 0), rank) for r in ranks]
        self.down, self.up = down.to(t).to(DEV), up.to(t).to(DEV)
        for a, r in enumerate(ranks_used):                       # behind an adapter's rank there may be anything
            self.down[a, :, r:], self.up[a, :, r:] = float("nan"), float("inf")
            down[a, :, r:], up[a, :, r:] = 0, 0
        self.ref_down, self.ref_up = down.to(t).double(), up.to(t).double()
        self.scale = (torch.randint(1, 4, (n_adapters,), generator=gen).float() / (2 if whole else 5)).to(DEV) if scale else None
        self.ranks = None if ranks is None else torch.tensor(ranks, dtype=torch.int32, device=DEV)
        px, pb, py = pads
        self.x = values(self.total, width + px).to(t).to(DEV)
        self.base = values(self.total, all_cols + pb, most=50).to(t).to(DEV)
        self.y = torch.full((self.total, all_cols + py), -7.0, dtype=t, device=DEV)
        self.adapter, self.rows = np.asarray(adapter), np.asarray(rows)
        self.pool = pool(typ)
        self.order, self.items = group(self.pool, self.adapter, self.rows, n_adapters, spare=spare)
        self.ad = B.make_adapters(down=self.down, up=self.up, n_adapters=n_adapters, rank=rank, width=width, part_cols=cols, scale=self.scale,
                                  ranks=self.ranks)
        size = self.pool.odma_adapt_scratch_bytes(self.ad, len(self.items))
        self.scratch = torch.full((size,), 0xff, dtype=torch.uint8, device=DEV)

    def run(self, stream=None, base=None, y=None):
        base, y = self.base if base is None else base, self.y if y is None else y
        self.pool.odma_adapt_rows(self.total, self.ad, len(self.items), self.items, self.order, self.x, self.x.stride(0), base, base.stride(0), y,
                                  y.stride(0), self.scratch, stream)
        return self

    def check(self, y=None):
        torch.cuda.synchronize()
        y = (self.y if y is None else y).cpu()
        which = torch.tensor(np.repeat(self.adapter, self.rows))
        has = (which >= 0) & (which < self.n_adapters)
        assert (y[~has] == -7).all() and (y[:, self.all_cols:] == -7).all()
        x, base = self.x[:, :self.width].cpu().double(), self.base[:, :self.all_cols].cpu().double()
        for a in sorted(set(which[has].tolist())):
            rows = which == a
            s = float(self.scale[a]) if self.scale is not None else 1.0
            at = 0
            for p, c in enumerate(self.cols):
                dn, up = self.ref_down[a, p], self.ref_up[a, at:at + c]
                h = x[rows] @ dn.T
                want = base[rows, at:at + c] + s * (h @ up.T)
                got = y[rows, at:at + c].double()
                if self.whole:
                    assert h.abs().max() < 2 ** 16 / 3 and want.abs().max() < 2 ** 22    # (sums and h are exact)
                    assert torch.equal(got, want.to(TYPE[self.typ]).double()), (a, p, (got - want).abs().max())
                else:
                    # sums of fp32 products: a step (2^-23, cut off or rounded) of what has been added up, for every term; h in bf16
                    # rows to 16 bits
                    step = 2.0 ** -23
                    loose_h = x[rows].abs() @ dn.abs().T * self.width * step + (2.0 ** -16 * h.abs() if self.typ == "bf16" else 0)
                    loose = s * (loose_h @ up.abs().T) + (2 * self.rank + 4) * step * (base[rows, at:at + c].abs() + s * (h.abs() @ up.abs().T))
                    half = torch.finfo(TYPE[self.typ]).eps / 2
                    assert ((got - want).abs() <= half * want.abs() + loose).all(), (got - want).abs().max()
                    # and far nearer than that on the whole: errors of so many terms mostly cancel
                    assert (got - want).norm() <= (half + 64 * step) * (want.norm() + (s * h.abs() @ up.abs().T).norm())
                at += c
        return self


SHAPES = [
    # rows of every request, adapters, width, columns, rank
    ([1], 1, 64, [16], 8),
    ([1] * 20, 20, 512, [48, 16], 16),
    ([1] * 70, 3, 1000, [336], 8),
    ([1] * 130, 2, 3584, [3584, 512, 512], 16),
    ([17, 40, 64, 65, 1, 200], 4, 520, [128, 64], 24),
    ([300, 5, 129], 2, 2056, [80, 16, 32, 1040], 32),
    ([64, 64], 1, 72, [64], 64),
    ([33, 90], 3, 136, [208], 128),
    ([5, 70], 2, 264, [96], 256),
    ([1, 2, 3, 0, 5], 4, 8, [16, 32], 8),
    # items of several runs of 16 rows, and more items than a wave has lanes, in the launch for few rows
    ([17, 40, 64, 65, 1, 200, 33], 4, 520, [1104, 64], 16),
    ([1, 2, 3] * 70, 200, 264, [64, 4112], 8),
    ([2] * 100, 9, 2056, [528, 32], 32),
    ([3] * 50, 60, 1032, [1040], 64),
]


@pytest.mark.parametrize("typ", ["bf16", "f32"])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_products(shape, typ):
    rows, n_adapters, width, cols, rank = SHAPES[shape]
    rng = np.random.default_rng(shape)
    adapter = np.arange(len(rows)) % n_adapters if shape < 2 else rng.integers(0, n_adapters, len(rows))
    for whole in (True, False):
        Case(typ, adapter, rows, n_adapters, width, cols, rank, whole=whole, seed=shape, scale=shape % 3 != 0).run().check()


@pytest.mark.parametrize("typ", ["bf16", "f32"])
def test_many_items(typ):
    """So many that no channels are cut, with rows of requests without an adapter between them and strides of their own."""
    rng = np.random.default_rng(3)
    rows = rng.integers(0, 150, 900)
    adapter = rng.integers(-1, 5, 900)
    c = Case(typ, adapter, rows, 5, 1032, [96, 32], 16, pads=(8, 16, 24))
    assert len(c.items) > 700
    c.run().check()


@pytest.mark.parametrize("typ", ["bf16", "f32"])
@pytest.mark.parametrize("rank", [8, 48])
def test_long_calls(rank, typ):
    """Rows that pass by the caches, in whole chunks of columns."""
    rng = np.random.default_rng(4)
    rows = rng.integers(0, 150, 300)
    c = Case(typ, rng.integers(-1, 6, 300), rows, 6, 264, [1040, 512], rank, pads=(8, 16, 24))
    assert c.total > 10000 and len(c.items) * 1552 / 512 >= 1024
    c.run().check()


@pytest.mark.parametrize("typ", ["bf16", "f32"])
@pytest.mark.parametrize("cols,rank,pads", [((1024, 512), 8, (8, 0, 64)), ((1024, 512), 48, (0, 64, 0)), ((64, 2048), 64, (0, 0, 0)), ((80, 2000), 64, (0, 0, 0)),
                                            ((64, 1984), 160, (16, 128, 64))])
def test_long_calls_of_groups(cols, rank, pads, typ):
    """The same in whole lines and not, with ranks of one group and of several, which neighbouring items share; the last block of them is not whole."""
    rng = np.random.default_rng(5)
    rows = rng.integers(0, 150, 320)
    c = Case(typ, rng.integers(-1, 7, 320), rows, 7, 72, list(cols), rank, pads=pads)
    assert c.total > 10000 and len(c.items) * sum(cols) / 512 >= 1024 and len(c.items) % 32
    c.run().check()


@pytest.mark.parametrize("typ", ["bf16", "f32"])
@pytest.mark.parametrize("rank,width,rows", [(64, 8200, [3, 20, 1, 64, 70]), (40, 8200, [1, 0, 2, 7, 100]), (8, 2056, [5000, 1, 3000, 130, 900]), (16, 1544, [5000, 1, 3000, 130, 900]),
                                             (24, 1544, [9000, 63, 64, 65, 1])])
def test_cut_channels(rank, width, rows, typ):
    """Two launches, of which the first cuts the channels between work-groups."""
    for whole in (True, False):
        Case(typ, [2, 0, 3, 2, 1], rows, 4, width, [48, 80], rank, seed=rank, whole=whole).run().check()


@pytest.mark.parametrize("typ", ["bf16", "f32"])
@pytest.mark.parametrize("rank", [8, 16, 24, 32, 40, 56, 64, 72, 96, 120, 128, 136, 256])
def test_ranks(rank, typ):
    """Every way in which ranks fill operands, with few rows and many."""
    for rows in ([3, 20, 1, 64, 70], [300, 1, 2900, 33, 129]):
        c = Case(typ, [2, 0, 3, 2, 1], rows, 4, 136, [48, 144], rank, seed=rank)
        c.run().check()
    Case(typ, [2, 0, 3, 2, 1], [3, 20, 1, 64, 70], 4, 136, [48, 144], rank, seed=rank, whole=False).run().check()


@pytest.mark.parametrize("typ", ["bf16", "f32"])
def test_ragged_ranks(typ):
    """Weights behind an adapter's rank are NaN and infinities here, and are not there."""
    for rank, ranks in ((16, [16, 8, 0, -3, 99, 9]), (64, [8, 64, 40, 1, 24, 33])):
        for whole, more in ((True, 1), (False, 1), (True, 60)):
            Case(typ, np.arange(12) % 6, [3 * more, 1, 70, 2, 9, 20] * 2, 6, 328, [64, 48], rank, ranks=ranks, whole=whole).run().check()


@pytest.mark.parametrize("typ", ["bf16", "f32"])
def test_in_place_and_slices(typ):
    c = Case(typ, [0, -1, 1, 0], [3, 2, 80, 1], 2, 256, [64, 32], 16, pads=(64, 32, 32))
    c.run().check()
    y = c.base.clone()
    c.run(base=y, y=y)
    torch.cuda.synchronize()
    has = torch.tensor(np.repeat(c.adapter, c.rows) >= 0)
    assert torch.equal(y[has][:, :96], c.y[has][:, :96]) and torch.equal(y[~has], c.base[~has]) and torch.equal(y[:, 96:], c.base[:, 96:])


def test_lists_that_name_nothing():
    """Items without an adapter that is there, rows outside x: skipped.  A NaN row stays in its row."""
    c = Case("bf16", [0, 1, 0], [5, 60, 9], 2, 256, [64], 8)
    c.run().check()
    want = c.y.clone()
    c.items[:, 0] = torch.where(c.items[:, 0] == 1, 2, c.items[:, 0])
    c.order[c.order == 2] = c.total
    c.order[c.order == 3] = -5
    c.y.fill_(-7)
    c.run()
    torch.cuda.synchronize()
    want[5:65], want[2:4] = -7, -7
    assert torch.equal(c.y, want)
    c = Case("bf16", [0, 1, 0], [5, 60, 9], 2, 256, [64], 8)
    # ... and an inner sum beyond fp32 is infinite behind weights that are not 0, not NaN
    c.down[0, 0, 1:, 5:7], c.down[0, 0, 0, 5:7], c.x[66], c.x[66, 5:7], c.x[7, 3] = 0, 1, 0, 3e38, float("nan")
    c.x[[r for r in range(c.total) if r != 66], 5:7] = 0
    c.run()
    torch.cuda.synchronize()
    want = c.y.clone()
    c.x[7, 3], c.x[66, 5:7] = 1, 0
    c.run()
    torch.cuda.synchronize()
    want, c.y = c.y, want
    torch.cuda.synchronize()
    rest = [r for r in range(c.total) if r not in (7, 66)]
    assert torch.equal(c.y[rest], want[rest]) and torch.isnan(c.y[7]).all()
    assert (torch.isinf(c.y[66]) == (c.up[0, :, 0] != 0)).all()


@pytest.mark.parametrize("typ", ["bf16", "f32"])
@pytest.mark.parametrize("rank", [16, 72])
def test_lists_of_more_rows(rank, typ):
    """Lists made for more rows than a call has: those that it has are adapted, wherever in the lists they stand."""
    n = 400
    adapter = np.arange(n)[::-1] % 350
    c = Case(typ, adapter, [1] * n, 350, 264, [64, 48], rank)
    whole = c.run().check().y.clone()
    for rows in (1, 17, 100):
        c.y.fill_(-7)
        c.pool.odma_adapt_rows(rows, c.ad, len(c.items), c.items, c.order, c.x, c.x.stride(0), c.base, c.base.stride(0), c.y, c.y.stride(0), c.scratch)
        torch.cuda.synchronize()
        assert torch.equal(c.y[:rows], whole[:rows]) and (c.y[rows:] == -7).all()


def test_far_rows():
    """Rows whose elements lie past 2^31."""
    c = Case("bf16", [0, 1], [2, 3], 2, 64, [32], 8)
    stride = 1 << 29
    far = [torch.zeros(5 * stride, dtype=torch.bfloat16, device=DEV).view(5, stride) for _ in range(2)]
    far[0][:, :64], far[1][:, :32] = c.x, c.base
    y = far[1]
    c.pool.odma_adapt_rows(5, c.ad, len(c.items), c.items, c.order, far[0], stride, y, stride, y, stride, c.scratch)
    c.check(y[:, :32].contiguous())


def test_streams_and_captured_calls():
    a, b = (Case("bf16", [0, 1, 2, -1, 1], [1, 9, 200, 4, 70], 3, 1024, [128, 64], 16, seed=s, whole=False) for s in (1, 2))
    want = []
    for c in (a, b):
        c.run()
        torch.cuda.synchronize()
        want.append(c.y.clone())
        c.y.fill_(-7)
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        a.run(one), b.run(two)
    torch.cuda.synchronize()
    assert torch.equal(a.y, want[0]) and torch.equal(b.y, want[1])
    # lists and products captured together; adapters and rows change between replays
    p, n = a.pool, len(a.adapter)
    ad = torch.tensor(a.adapter, dtype=torch.int32, device=DEV)
    rs = torch.tensor(np.concatenate([[0], np.cumsum(a.rows)]), dtype=torch.int64, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.odma_group_adapters(n, ad, 3, rs, a.total, a.order, len(a.items), a.items)
        a.run()
    for i in range(4):
        a.adapter = np.array([[0, 1, 2, -1, 1], [2, 2, 2, 2, 2], [-1, 0, -1, 1, 0], [-1] * 5][i])
        ad.copy_(torch.tensor(a.adapter, dtype=torch.int32))
        a.y.fill_(-7)
        a.scratch.fill_(85 * i)
        graph.replay()
        a.check()
        if i == 0:
            assert torch.equal(a.y, want[0])
