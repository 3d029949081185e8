"""The calls on a batch's rows around the attention at the ends of their ranges."""
import math

import numpy as np
import pytest
import torch

from paper_2512_09427_amd import binding as B
from tests import test_gpu_adapters as adapters
from tests import test_gpu_add_norm as norms
from tests import test_gpu_score_tokens as scores

DEV = "cuda"
pytestmark = pytest.mark.gpu
TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
FEW, MANY = [3, 20, 1, 64, 70], [300, 1, 2900, 33, 129]


# ---- adapters

@pytest.mark.parametrize("typ", ["bf16", "f32"])
@pytest.mark.parametrize("rank", [8, 16, 24, 32, 48, 64, 72, 96, 128, 136, 168, 256])
@pytest.mark.parametrize("rows", [FEW, MANY])
def test_inner_sums_keep_all_bits(rows, rank, typ):
    """Pairs of ranks whose inner sums, whole numbers of 20 bits, differ by a channel of x, one added and one subtracted."""
    gen = torch.Generator().manual_seed(rank)
    c = adapters.Case(typ, [2, 0, 3, 2, 1], rows, 4, 64, [48, 144], rank, seed=rank, scale=False)
    t = TYPE[typ]
    x = torch.randint(64, 128, c.x.shape, generator=gen).float()
    down = torch.randint(64, 127, (4, 2, rank, 64), generator=gen).float()
    down[:, :, 1::2] = down[:, :, ::2]
    channel = torch.randint(0, 64, (4, 2, rank // 2, 1), generator=gen)
    down[:, :, 1::2] += torch.zeros(4, 2, rank // 2, 64).scatter_(3, channel, 1.0)
    up = torch.zeros(4, 192, rank)
    for _ in range(2):
        pair = torch.randint(0, rank // 2, (4, 192, 1), generator=gen)
        sign = torch.randint(0, 2, (4, 192, 1), generator=gen) * 2.0 - 1
        up.scatter_(2, 2 * pair, sign).scatter_(2, 2 * pair + 1, -sign)
    c.x.copy_(x.to(t)), c.down.copy_(down.to(t)), c.up.copy_(up.to(t))
    c.run()
    torch.cuda.synchronize()
    y = c.y.cpu()
    for r, (a, start) in enumerate(zip(c.adapter, np.cumsum(rows) - rows)):
        mine = slice(int(start), int(start) + rows[r])
        for p, (lo, hi) in enumerate(((0, 48), (48, 192))):
            h = x[mine].double() @ down[a, p].double().T
            assert (h.abs() @ up[a, lo:hi].double().abs().T).max() < 2 ** 22 and h.max() > 2 ** 18    # (sums are exact, also of their quarters)
            want = c.base[mine, lo:hi].cpu().double() + h @ up[a, lo:hi].double().T
            assert torch.equal(y[mine, lo:hi], want.to(t)), (r, p, (y[mine, lo:hi].double() - want).abs().max())


@pytest.mark.parametrize("total,cols", [([3, 20, 1, 64], [64, 48]), ([150] * 300, [1024, 576])])
def test_rows_of_fp8_pools(total, cols):
    """They are bf16: few of them, and more than the caches keep, in lines that are whole."""
    c = adapters.Case("bf16", np.arange(len(total)) % 4, total, 4, 264, cols, 16)
    kv = torch.zeros(80 * 128, dtype=torch.uint8, device=DEV)
    c.pool = B.Pool(*B.make_config(n_layers=1, n_q_heads=1, n_kv_heads=1, head_dim=128, kv_dtype=B.FP8, out_dtype=B.BF16, main_tokens=64, safety_tokens=16,
                                   large_cap=16, boundaries=(16,), quantiles=((1, 2),), max_requests=8, k_pool=kv, v_pool=kv.clone()))
    assert c.pool.odma_adapt_scratch_bytes(c.ad, len(c.items)) == c.scratch.numel()
    c.run().check()


@pytest.mark.parametrize("typ", ["bf16", "f32"])
@pytest.mark.parametrize("rank", [8, 16, 24, 64, 72, 136])
@pytest.mark.parametrize("rows", [FEW, MANY])
def test_infinite_weights(rows, rank, typ):
    """An infinite weight of up gives what the formula gives: infinities of the inner sum's sign, NaN behind a sum of 0 and between
    infinities of both signs."""
    c = adapters.Case(typ, [2, 0, 3, 2, 1], rows, 4, 64, [48, 144], rank, seed=rank)
    c.up[0, 5, 3], c.up[2, 100, rank - 1], c.up[2, 100, 0], c.up[3, 7, 2], c.up[1, 150, rank // 2] = math.inf, math.inf, -math.inf, -math.inf, math.inf
    c.x[4, 9], c.x[30, 8] = math.inf, -math.inf
    c.run()
    torch.cuda.synchronize()
    x, y, up, seen = c.x.cpu().double(), c.y.cpu().float(), c.up.cpu().double(), 0
    for r, (a, start) in enumerate(zip(c.adapter, np.cumsum(rows) - rows)):
        mine = slice(int(start), int(start) + rows[r])
        for p, (lo, hi) in enumerate(((0, 48), (48, 192))):
            h = (x[mine, None] * c.ref_down[a, p]).sum(-1)                          # (products one by one: 0 x inf is NaN)
            want = c.base[mine, lo:hi].cpu().double() + float(c.scale[a]) * (h[:, None] * up[a, None, lo:hi]).sum(-1)
            want, got = want.to(TYPE[typ]).float(), y[mine, lo:hi]
            seen += int(torch.isinf(want).sum())
            assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got.nan_to_num(nan=0.0), want.nan_to_num(nan=0.0))
    assert seen > 50


def lists_of(adapter, start, n_adapters, max_rows, max_items):
    """The lists, for any number of rows."""
    order, items = np.full(max_rows, -1), np.tile(np.array([B.ADAPTER_NONE, 0, 0, 0]), (max_items, 1))
    at, seen = 0, 0
    for a in range(n_adapters):
        first, some = at, False
        for r in np.flatnonzero(adapter == a):
            some = some or start[r + 1] > start[r]
            row = np.arange(start[r], start[r] + min(start[r + 1] - start[r], max_rows - at))
            order[at:at + len(row)] = np.where(row < 2 ** 31, row, -1)
            at += len(row)
        for f in range(first, at, 64):
            items[first // 64 + seen + (f - first) // 64] = a, f, min(64, at - f), 0
        seen += some
    return order, items


ROWS = [[1 << 27] * 70, [100, 1 << 40, 3, 0, 5] * 9, [300] + [0] * 9 + [(1 << 31) - 301, 7, 1 << 32, 9, (1 << 27) - 1], [1 << 22] * 1500, [5, 1 << 27, 1 << 27] * 60]


@pytest.mark.parametrize("rows,max_rows", [(r, m) for r in ROWS for m in (1, 63, 1000, 70001)] + [(ROWS[0], 1 << 26), (ROWS[3], 4000001), (ROWS[4], 30000000)])
def test_lists_of_more_rows_than_32_bits_count(rows, max_rows):
    """Also with lists so long that sums of what fits into them are beyond 32 bits."""
    n = len(rows)
    start = np.concatenate([[0], np.cumsum(np.array(rows, np.int64))])
    p, rng = adapters.pool(), np.random.default_rng(n)
    for adapter in (np.arange(n) // 33, (np.arange(n) < 34).astype(np.int64), rng.integers(-1, 5, n))[:3 if max_rows < 1 << 17 else 2]:
        n_adapters = int(adapter.max()) + 1
        max_items = max_rows // 64 + min(n, n_adapters) + 2
        order = torch.full((max_rows + 8,), 77, dtype=torch.int32, device=DEV)
        items = torch.full((max_items + 2, 4), 77, dtype=torch.int32, device=DEV)
        ad, rs = torch.tensor(adapter, dtype=torch.int32, device=DEV), torch.tensor(start, device=DEV)
        p.odma_group_adapters(n, ad, n_adapters, rs, max_rows, order, max_items, items)
        want = [torch.from_numpy(w).to(DEV) for w in lists_of(adapter, start, n_adapters, max_rows, max_items)]
        assert torch.equal(order[:max_rows].long(), want[0]) and torch.equal(items[:max_items].long(), want[1])
        assert (order[max_rows:] == 77).all() and (items[max_items:] == 77).all()


# ---- scores

def check_parts_with_nothing_on(rest, typ):
    vocab = 131072
    for on in (slice(70000, None), slice(0, 30), slice(40000, 40001)):
        x = torch.full((2, vocab), -math.inf)
        x[0, on] = rest
        x[1, on] = rest * torch.linspace(0.5, 1, len(x[1, on]))
        scores.Call(x.to(TYPE[typ]).float(), typ, vocab, [on.start, on.start], 9).run().check()


@pytest.mark.parametrize("typ", ["bf16", "f32"])
@pytest.mark.parametrize("rest", [-3.38e38, -5e30, -1e3, 2.0, 1e3])
def test_parts_with_nothing_on(rest, typ):
    """Whole parts of a row are switched off; what is on is far below 0, or above it."""
    check_parts_with_nothing_on(rest, typ)


def logits_with(fill, vocab, typ):
    """Rows with `fill` in some places, in all, or nearly all."""
    x = scores.some(8, vocab, typ, seed=vocab)
    x[0, : vocab // 2] = fill
    x[1, :] = fill
    x[1, [0, vocab // 3, vocab - 1]] = torch.tensor([1.0, 2.0, 0.5])
    x[2] = fill
    x[3, ::2] = fill
    x[4, :4096] = fill
    x[5, vocab // 2] = fill
    x[6] = fill * (1 + torch.rand(vocab, generator=torch.Generator().manual_seed(1)) / 2)
    x[7, :] = -math.inf
    x[7, vocab // 2:] = fill
    return x.to(TYPE[typ]).float()


@pytest.mark.parametrize("typ", ["bf16", "f32"])
@pytest.mark.parametrize("fill", [-6e4, -1e6, -1e9, -1e10, -1e20, -1e30, -3.38e38, 1e6, 3e7, 1e10, 1e20, 1e29, 1e31, 1e38])
@pytest.mark.parametrize("vocab", [9, 4099, 40009])             # (the last is cut into parts)
def test_logits_far_from_0(vocab, fill, typ):
    for scale in (1.0, 2.0 ** -24, 1e5, 2.0 ** 24):
        tokens = [0, vocab // 3, vocab - 1, 2, 1, vocab // 2, 3, vocab - 1]
        scores.Call(logits_with(fill, vocab, typ), typ, vocab, tokens, 5, scale=scale).run().check()


@pytest.mark.parametrize("typ", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [300, 700])                    # eight waves of a work-group, and four
def test_many_rows_far_from_0(rows, typ):
    vocab = 2501
    x = torch.cat([logits_with(f, vocab, typ) for f in (-1e4, -1e9, -1e30, 1e10, 1e30)]).repeat(rows // 40 + 1, 1)[:rows]
    scores.Call(x, typ, vocab, [37 * r % vocab for r in range(rows)], 5).run().check()


@pytest.mark.parametrize("typ", ["bf16", "f32"])
@pytest.mark.parametrize("rest", [-1e30, -1e20, -1e9, 1e9, 1e10])
def test_parts_with_nothing_on_far_from_0(rest, typ):
    check_parts_with_nothing_on(rest, typ)


@pytest.mark.parametrize("rows,vocab", [(6, 40009), (600, 3001)])   # cut into parts, whole
def test_rows_that_are_not_there_have_no_logits(rows, vocab):
    """The tensor of logits ends with the last row that is there; tokens of the others may be any."""
    x = scores.some(rows, vocab, "bf16", seed=5)
    slots = torch.full((rows,), B.SLOT_NONE, dtype=torch.int64, device=DEV)
    slots[0], slots[2] = 0, 5
    for top in (0, 6):
        c = scores.Call(x, "bf16", vocab, [r % vocab for r in range(rows)], top, slots=slots)
        c.logits = c.logits[:3 * vocab].clone()
        c.run().check()


# ---- residual rows

@pytest.mark.parametrize("typ,res", norms.TYPES)
@pytest.mark.parametrize("rows,width", [(5, 512), (5, 1000), (5, 2048), (6, 3584), (3, 8192), (2, 16384), (2, 32768), (16400, 520), (1030, 8192), (49170, 2056)])
def test_squares_that_add_up_beyond_fp32(rows, width, typ, res):
    """Rows whose mean square is within fp32's range and whose sum of squares is not, beside others."""
    def edit(blk, old):
        blk[::2] *= 2e18
        old[::2] *= 1e18
    for post in (False, True):
        if not post or rows < 20000:
            norms.Case(typ, res, rows, width, post=post, seed=width, edit=edit).run().check()
    norms.Case(typ, res, rows, width, block=False, eps=0.0, edit=edit).run().check()


@pytest.mark.parametrize("width", [8200, 16392])
def test_as_many_rows_as_a_call_takes(width):
    """2^22 rows of more channels than eight waves take at a time; most of them are not there."""
    rows, at = 1 << 22, [0, 1, 77777, (1 << 22) - 1]
    c = norms.Case("bf16", "bf16", 1, width, gate="sigmoid", one_gate=True, seed=width)
    slots = torch.full((rows,), B.SLOT_NONE, dtype=torch.int64, device=DEV)
    slots[at] = 0
    x = torch.empty(rows, width, dtype=torch.bfloat16, device=DEV)
    x[:2000], x[-2000:] = -7, -7
    # one block, gate and residual for all rows; it is not kept
    c.pool.odma_add_norm(rows, c.how, c.block, 0, c.old, 0, slots, None, x)
    torch.cuda.synchronize()
    c.x.copy_(x[:1])
    c.check(keep=False)
    assert all(torch.equal(x[r], x[0]) for r in at) and (x[2:2000] == -7).all() and (x[-2000:-1] == -7).all()
    del x
    torch.cuda.empty_cache()
