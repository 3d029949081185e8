"""odma_build_tables against the definition written out in Python: whole numbers, so every one has to be equal."""
import numpy as np
import pytest
import torch

from paper_2512_09427_amd import binding as B

DEV = "cuda"
pytestmark = pytest.mark.gpu


def pool(max_requests=4096):
    args = dict(n_layers=1, n_q_heads=2, n_kv_heads=1, head_dim=64, kv_dtype=B.BF16, out_dtype=B.BF16, main_tokens=64, safety_tokens=64,
                large_cap=64, boundaries=(64,), quantiles=((1, 2),), max_requests=max_requests)
    k = torch.zeros(128 * 64, dtype=torch.bfloat16, device=DEV)
    return B.Pool(*B.make_config(**args, k_pool=k, v_pool=torch.zeros_like(k)))


def expected(lengths, n_new, offsets, start, poff, plen, stride, max_rows):
    n = len(lengths)
    table = np.zeros((n, stride), np.int32)
    row_start, pos, slot = [0], [], []
    for r in range(n):
        group = [p for p in range(len(plen)) if start[p] <= r < start[p + 1]]
        shared = max(int(plen[group[-1]]), 0) // 16 * 16 if group else 0
        where = [int(poff[group[-1]]) + t if t < shared else int(offsets[r]) + t - shared for t in range(max(lengths[r], 0))]
        for j in range(min(stride, (len(where) + 15) // 16)):
            table[r, j] = where[16 * j] // 16
        new = min(max(n_new[r], 0), len(where)) if n_new is not None else min(len(where), 1)
        for t in range(len(where) - new, len(where)):
            pos.append(t)
            slot.append(-2 if t < shared else where[t])
        row_start.append(len(pos))
    pos, slot = (pos + [0] * max_rows)[:max_rows], (slot + [-1] * max_rows)[:max_rows]
    return table, np.array(row_start, np.int64), np.array(pos, np.int32), np.array(slot, np.int64)


def build(p, lengths, n_new, offsets, start, poff, plen, stride, max_rows, guard=64, skip=()):
    n = len(lengths)
    dev = lambda a, t: None if a is None else torch.tensor(np.asarray(a), dtype=t, device=DEV)  # noqa: E731
    outs = [torch.full((size + guard,), -77, dtype=t, device=DEV)
            for size, t in ((n * stride, torch.int32), (n + 1, torch.int64), (max_rows, torch.int32), (max_rows, torch.int64))]
    given = [None if i in skip else o for i, o in enumerate(outs)]
    np_ = len(plen)
    p.odma_build_tables(n, dev(lengths, torch.int32), dev(n_new, torch.int32), dev(offsets, torch.int64), np_,
                        dev(start, torch.int32) if np_ else None, dev(poff, torch.int64) if np_ else None,
                        dev(plen, torch.int32) if np_ else None, given[0], 0 if given[0] is None else stride, max_rows, *given[1:])
    got = [o.cpu().numpy() for o in outs]
    for i, g in enumerate(got):
        size = g.size - guard
        assert (g[size if i not in skip else 0:] == -77).all(), f"output {i} was written behind its end"
    return got[0][:n * stride].reshape(n, stride), got[1][:n + 1], got[2][:max_rows], got[3][:max_rows]


# name -> lengths, n_new, prefix_start, prefix_lengths, stride, max_rows
CASES = {
    "one token": ([1], None, [0], [], 1, 1),
    "one request": ([1777], None, [0], [], 112, 3),
    "an empty place": ([0], None, [0], [], 3, 2),
    "ragged step": ([1, 16, 17, 0, 4095, 33], None, [0], [], 256, 6),
    "prompts": ([5, 100, 1, 0, 16, 31, 1500], [5, 100, 1, 0, 16, 31, 1500], [0], [], 94, 1700),
    "chunks and odd numbers": ([40, 100, 7, 9], [10, 200, -3, 0], [0], [], 7, 150),
    "fewer rows than there are": ([40, 100, 7], [40, 100, 7], [0], [], 7, 60),
    "fewer entries than blocks": ([40, 1000, 7], None, [0], [], 2, 3),
    "one prefix": ([40, 100, 1000, 17], [8, 100, 990, 1], [0, 4], [33], 64, 1200),
    "groups, places outside them": ([40, 100, 0, 64, 65, 7, 300, 20], [1, 2, 3, 4, 65, 7, 100, 20], [1, 3, 3, 6], [48, 500, 64], 20, 250),
    "prefixes below a block": ([20, 20, 20, 20], [20, 1, 20, 0], [0, 1, 2, 4], [15, 0, -5], 2, 64),
    "a request shorter than its prefix": ([10, 200], [10, 200], [0, 2], [160], 13, 210),
}


@pytest.mark.parametrize("skip", [(), (0,), (1, 2), (0, 1, 3), (2, 3)], ids=str)
@pytest.mark.parametrize("name", list(CASES))
def test_against_the_definition(name, skip):
    lengths, n_new, start, plen, stride, max_rows = CASES[name]
    rng = np.random.default_rng(3)
    offsets, poff = rng.integers(0, 1 << 30, len(lengths)) * 16, rng.integers(0, 1 << 30, len(plen)) * 16
    args = (lengths, n_new, offsets, start, poff, plen, stride, max_rows)
    for i, (g, e) in enumerate(zip(build(pool(), *args, skip=skip), expected(*args))):
        if i not in skip:
            np.testing.assert_array_equal(g, e, err_msg=f"{name}, output {i}")


@pytest.mark.parametrize("n,mid,prefixes", [(64, 30, 3), (1023, 20, 0), (1024, 20, 7), (1025, 20, 400), (3001, 9, 1), (1, 70000, 1), (3, 40000, 2)])
def test_random_batches(n, mid, prefixes):
    """Beyond 1024 requests a work-group has several; beyond a thousand rows or entries a request has several work-groups."""
    rng = np.random.default_rng(n)
    lengths = rng.integers(0, 2 * mid, n)
    n_new = rng.integers(0, 2 * mid, n)
    start = np.sort(rng.integers(0, n + 1, prefixes + 1))
    plen = rng.integers(0, mid, prefixes)
    offsets, poff = rng.integers(0, 1 << 30, n) * 16, rng.integers(0, 1 << 30, prefixes) * 16
    total = int(np.minimum(lengths, n_new).sum())
    args = (lengths, n_new, offsets, start, poff, plen, 2 * mid // 16 + 1, total + 1000)
    for g, e in zip(build(pool(), *args), expected(*args)):
        np.testing.assert_array_equal(g, e)


def test_slots_past_32_bits():
    """Offsets of a pool of more than 2^32 tokens (block numbers fit 32 bits)."""
    offsets, poff = [(1 << 34) + 16, (1 << 34) + 1600], [1 << 33]
    args = ([100, 50], [100, 50], offsets, [0, 2], poff, [32], 8, 160)
    for g, e in zip(build(pool(), *args), expected(*args)):
        np.testing.assert_array_equal(g, e)


def test_captured_and_replayed_on_lengths_that_grow():
    p = pool()
    n, stride, rows = 37, 64, 48
    rng = np.random.default_rng(1)
    lengths, offsets, plen = rng.integers(0, 900, n), rng.integers(0, 1000, n) * 16, [100]
    dev = lambda a, t: torch.tensor(np.asarray(a), dtype=t, device=DEV)  # noqa: E731
    L, O, S, PO, PL = dev(lengths, torch.int32), dev(offsets, torch.int64), dev([3, 30], torch.int32), dev([16000], torch.int64), dev(plen, torch.int32)
    outs = (torch.zeros(n, stride, dtype=torch.int32, device=DEV), torch.zeros(n + 1, dtype=torch.int64, device=DEV),
            torch.zeros(rows, dtype=torch.int32, device=DEV), torch.zeros(rows, dtype=torch.int64, device=DEV))
    call = lambda: p.odma_build_tables(n, L, None, O, 1, S, PO, PL, outs[0], stride, rows, *outs[1:])  # noqa: E731
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        call()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for step in range(4):
        graph.replay()
        torch.cuda.synchronize()
        for g, e in zip(outs, expected(L.cpu().numpy(), None, offsets, [3, 30], [16000], plen, stride, rows)):
            np.testing.assert_array_equal(g.cpu().numpy(), e)
        L += torch.where(L > 0, 5 * step + 1, step % 2).int()
