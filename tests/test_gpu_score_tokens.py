"""odma_score_tokens against log-softmax, entropy and sorted order in 64 bits: vocabularies from one token on, rows that begin at
any element, rows cut into parts and whole, tokens switched off, infinities, NaN, equal and ordered logits, tokens and rows that
are not there, streams, captured calls."""
import math

import numpy as np
import pytest
import torch

from paper_2512_09427_amd import binding as B

DEV = "cuda"
pytestmark = pytest.mark.gpu
TYPE = {"f32": (torch.float32, B.F32), "bf16": (torch.bfloat16, B.BF16)}
FULL = -3.38e38                                                  # (finite in bf16 too)


def pool(tokens=64):
    kv = torch.zeros(2 * (tokens + 16) * 32, dtype=torch.bfloat16, device=DEV)
    return B.Pool(*B.make_config(n_layers=1, n_q_heads=2, n_kv_heads=2, head_dim=32, kv_dtype=B.BF16, out_dtype=B.BF16, main_tokens=tokens,
                                 safety_tokens=16, large_cap=16, boundaries=(16,), quantiles=((1, 2),), max_requests=1, k_pool=kv,
                                 v_pool=kv.clone()))


class Call:
    def __init__(self, logits, typ, vocab, tokens, top, *, scale=1.0, first=0, slots=None):
        """logits: [rows][stride] on the CPU, already rounded to the type; rows begin at element `first`."""
        self.typ, self.vocab, self.top, self.scale, self.slots = typ, vocab, top, scale, slots
        self.rows, self.stride = logits.shape
        self.held = logits.to(DEV)
        self.flat = torch.cat([torch.full((first,), 9e9), logits.flatten(), torch.full((64,), 9e9)]).to(TYPE[typ][0]).to(DEV)
        self.logits = self.flat[first:]
        self.tokens = torch.tensor(tokens, dtype=torch.int32, device=DEV)
        self.pool = pool()
        self.scratch = torch.empty(self.pool.odma_score_scratch_bytes(self.rows, vocab, top) + 256, dtype=torch.uint8, device=DEV).fill_(0xff)[:-256]
        self.clear()

    def clear(self):
        self.logprob, self.entropy = (torch.full((self.rows,), 77.0, device=DEV) for _ in range(2))
        self.rank = torch.full((self.rows,), -77, dtype=torch.int32, device=DEV)
        self.top_id = torch.full((self.rows, self.top), -77, dtype=torch.int32, device=DEV)
        self.top_logprob = torch.full((self.rows, self.top), 77.0, device=DEV)

    def run(self, stream=None):
        self.pool.odma_score_tokens(self.rows, self.logits, self.stride, TYPE[self.typ][1], self.vocab, self.scale, self.tokens, self.slots, self.top,
                                    self.logprob, self.rank, self.entropy, self.top_id if self.top else None,
                                    self.top_logprob if self.top else None, self.scratch, stream)
        return self

    def check(self):
        torch.cuda.synchronize()
        raw = self.held[:, :self.vocab].double().cpu().numpy()
        got = [t.cpu().numpy() for t in (self.logprob, self.rank, self.entropy, self.top_id, self.top_logprob)]
        for r in range(self.rows):
            if self.slots is not None and int(self.slots[r]) in (B.SLOT_NONE, 10 ** 9):
                assert got[0][r] == 77 and got[1][r] == -77 and got[2][r] == 77 and (got[3][r] == -77).all() and (got[4][r] == 77).all()
                continue
            self.check_row(raw[r], int(self.tokens[r]), [g[r] for g in got])

    def check_row(self, x, token, got):
        lp, rank, entropy, ids, lps = got
        real = 0 <= token < self.vocab
        # the largest: by logit, then by token, of those that are on (a NaN is none of them)
        on = np.flatnonzero(x > -np.inf)
        order = on[np.lexsort((on, -x[on]))][:self.top]
        assert list(ids[:len(order)]) == list(order) and (ids[len(order):] == B.TOKEN_NONE).all(), (ids, order)
        assert rank == ((x > x[token]).sum() if real else self.vocab)
        if np.isnan(x).any() or (x == np.inf).any():
            assert math.isnan(entropy) and (math.isnan(lp) if real else lp == -math.inf)
            assert np.isnan(lps[:len(order)]).all() and (lps[len(order):] == -math.inf).all()
            return
        if not len(on):
            assert entropy == 0 and lp == -math.inf and (lps == -math.inf).all()
            return
        m = x.max()
        with np.errstate(over="ignore"):
            d = (x - m) * self.scale
        e = np.exp(d)
        log_l = math.log(e.sum())
        p = e / e.sum()
        h = log_l - (p[p > 0] * d[p > 0]).sum()
        # fp32: sums of a lane's terms one after the other (a 256th of the row and the steps that join lanes, waves and parts),
        # each term off by a few steps and by those of its exponent; log and differences a step or two each
        sums = self.vocab / 256 + 64
        spread = (p * np.minimum(-d, 200)).sum()                    # what rounded exponents do to the sum
        tol = 2.0 ** -24 * (sums + 4 * spread + 4 * log_l)
        for i, g in ([(token, lp)] if real else []) + list(zip(order, lps)):
            want = d[i] - log_l
            if want < -3.4028234e38:                                # (beyond fp32)
                assert g == -math.inf
            else:
                assert abs(g - want) <= tol + 4 * 2.0 ** -24 * abs(d[i]), (g, want)
        assert real or lp == -math.inf
        assert (lps[len(order):] == -math.inf).all()
        assert abs(entropy - h) <= tol + 2.0 ** -24 * (sums + 8) * (1 + spread) + 8 * 2.0 ** -24 * (p[p > 0] * d[p > 0] ** 2).sum(), (entropy, h)


def some(rows, stride, typ, seed=0, size=3.0):
    gen = torch.Generator().manual_seed(seed)
    return (torch.randn(rows, stride, generator=gen) * size).to(TYPE[typ][0]).float()


@pytest.mark.parametrize("typ", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [1, 2, 7, 8, 9, 15, 63, 64, 65, 255, 513, 2047, 2048, 2049, 4099])
def test_small_vocabularies(vocab, typ):
    for top in sorted({0, 1, min(5, vocab), min(64, vocab)}):
        for first in (0, 1, 5):
            x = some(3, vocab + first % 3, typ, seed=vocab + top)
            Call(x, typ, vocab, [0, vocab - 1, vocab // 2], top, first=first).run().check()


@pytest.mark.parametrize("typ", ["bf16", "f32"])
@pytest.mark.parametrize("rows,vocab,top,scale", [(1, 128000, 20, 1.0), (2, 50001, 64, 0.7), (5, 32003, 5, 1.6), (17, 131072, 20, 1.0),
                                                  (300, 9001, 20, 1.0), (300, 40001, 20, 1.0), (1, 32768, 64, 1.0),
                                                  (16, 32769, 20, 1.0), (256, 20001, 20, 1.0), (700, 3001, 64, 2.5), (1025, 2500, 3, 1.0), (2, 262147, 1, 1.0)])
def test_parts_and_whole_rows(rows, vocab, top, scale, typ):
    x = some(rows, vocab + vocab % 2, typ, seed=rows)
    gen = torch.Generator().manual_seed(7)
    tokens = torch.randint(0, vocab, (rows,), generator=gen).tolist()
    tokens[0] = int(x[0, :vocab].argmax())
    Call(x, typ, vocab, tokens, top, scale=float(np.float32(scale)), first=1).run().check()


@pytest.mark.parametrize("typ", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [1, 1024])                      # cut into parts, whole
@pytest.mark.parametrize("order", ["up", "down", "equal", "two values", "zeros of both signs", "low", "steps"])
def test_ordered_and_equal_logits(order, rows, typ):
    vocab = 40011 if rows == 1 else 5003
    i = torch.arange(vocab, dtype=torch.float64)
    x = {"up": i / 128, "down": -i / 128, "equal": torch.full_like(i, -2.5), "two values": (i % 3 == 1).double(),
         "zeros of both signs": torch.where(i % 2 == 0, -0.0, 0.0), "low": torch.where(i % 7 == 3, i / 1000, FULL),
         "steps": torch.floor(i / 300) % 5}[order].to(TYPE[typ][0]).float()
    at = [0, vocab - 1, 5, 1234]
    rows_x = x[None].repeat(4 if rows == 1 else rows, 1)
    tokens = at if rows == 1 else [(37 * r) % vocab for r in range(rows)]
    for top in (1, 20, 64):
        c = Call(rows_x[:1] if rows == 1 else rows_x, typ, vocab, tokens[:1] if rows == 1 else tokens, top).run()
        if rows == 1:
            c.check()
            continue
        torch.cuda.synchronize()
        # rows of an odd length begin at eight places of a piece, which order a row's sums: those against the definition, the others,
        # which are like one of them in that too, against them
        for r in range(8):
            c.check_row(x.double().numpy(), tokens[r], [t[r].cpu().numpy() for t in (c.logprob, c.rank, c.entropy, c.top_id, c.top_logprob)])
        for t in (c.entropy, c.top_id, c.top_logprob):
            assert (t.view(128, 8, -1) == t[:8].view(1, 8, -1)).all()
        assert (c.rank.cpu() == (x[None] > x[torch.tensor(tokens)][:, None]).sum(1)).all()


@pytest.mark.parametrize("typ", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [9, 700, 40009])
def test_switched_off_infinite_and_nan(vocab, typ):
    x = some(16, vocab, typ, seed=3)
    x[0] = -math.inf
    x[1, 1:] = -math.inf
    x[2, :-1] = -math.inf
    x[3, ::2] = -math.inf
    x[4] = FULL
    x[5, :-2] = FULL
    x[6, 3] = math.nan
    x[7] = math.nan
    x[8, 4] = math.inf
    x[9, 2:5] = math.inf
    x[10, 1:] = math.nan
    x[11, :4] = -math.inf
    x[12] *= 1e-42
    x[13] = x[13].abs() * 1e36
    x[14, 1] = 3e38
    x[14, 2] = FULL
    x = x.to(TYPE[typ][0]).float()
    tokens = [0, 0, vocab - 1, 1, 2, vocab - 1, 2, 0, 4, 0, 0, 3, 5, 6, 2, B.TOKEN_NONE]
    for top in (0, 1, 7):
        Call(x, typ, vocab, tokens, top).run().check()
    tokens[3:7] = [vocab, -5, 2 ** 31 - 1, -2 ** 31]
    Call(x, typ, vocab, tokens, 3, scale=0.125).run().check()


def test_rows_that_are_not_there():
    x = some(40, 3000, "bf16")
    slots = torch.tensor([[-1, 0, 10 ** 9, 79, -2][r % 5] for r in range(40)], dtype=torch.int64, device=DEV)
    for rows in (1, 40):
        Call(x[:rows], "bf16", 3000, list(range(rows)), 6, slots=slots[:rows]).run().check()
        Call(x[:rows], "bf16", 3000, list(range(rows)), 6, slots=slots[1:rows + 1] if rows < 40 else slots).run().check()


def test_fewer_results():
    x = some(3, 10007, "f32", seed=8)
    c = Call(x, "f32", 10007, [5, 6, 7], 9).run()
    p = c.pool
    lp, ent, rank, ids, lps = (t.clone() for t in (c.logprob, c.entropy, c.rank, c.top_id, c.top_logprob))
    args = (3, c.logits, c.stride, B.F32, 10007, 1.0)
    c.clear()
    p.odma_score_tokens(*args, c.tokens, None, 0, c.logprob, None, None, None, None, c.scratch)
    assert torch.equal(c.logprob, lp) and (c.rank == -77).all() and (c.entropy == 77).all()
    p.odma_score_tokens(*args, None, None, 0, None, None, c.entropy, None, None, c.scratch)
    assert torch.equal(c.entropy, ent)
    p.odma_score_tokens(*args, None, None, 9, None, None, None, c.top_id, None, c.scratch)
    assert torch.equal(c.top_id, ids) and (c.top_logprob == 77).all()
    p.odma_score_tokens(*args, c.tokens, None, 9, None, c.rank, None, None, c.top_logprob, c.scratch)
    assert torch.equal(c.top_logprob, lps) and torch.equal(c.rank, rank)


@pytest.mark.parametrize("rows", [3, 1100])
def test_streams_and_captured_calls(rows):
    """Two calls at once with scratch of their own, and a captured one replayed on new logits: the same bits as a call by itself."""
    a = Call(some(rows, 6001, "bf16", seed=1), "bf16", 6001, [r % 6001 for r in range(rows)], 12)
    b = Call(some(rows, 6001, "bf16", seed=2), "bf16", 6001, [r % 6001 for r in range(rows)], 12)
    want = []
    for c in (a, b):
        c.run()
        torch.cuda.synchronize()
        want.append([t.clone() for t in (c.logprob, c.rank, c.entropy, c.top_id, c.top_logprob)])
        c.clear()
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        a.run(one)
        b.run(two)
    torch.cuda.synchronize()
    for c, w in zip((a, b), want):
        assert all(torch.equal(t, v) for t, v in zip((c.logprob, c.rank, c.entropy, c.top_id, c.top_logprob), w))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.run()
    keep = a.flat.clone()
    for i in range(4):
        for t in (a.logprob, a.entropy, a.top_logprob):
            t.fill_(-7)
        src, w = ((b.flat, want[1]), (keep, want[0]))[i % 2]
        a.flat.copy_(src)
        a.scratch.fill_(i * 85)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(t, v) for t, v in zip((a.logprob, a.rank, a.entropy, a.top_id, a.top_logprob), w))


def test_far_rows():
    """Rows whose elements lie past 2^31."""
    rows, stride, vocab = 5, 1 << 29, 3001
    flat = torch.zeros(rows * stride, dtype=torch.bfloat16, device=DEV)
    x = some(rows, vocab, "bf16", seed=4)
    flat.view(rows, stride)[:, :vocab] = x.to(DEV)
    c = Call(x, "bf16", vocab, [1, 2, 3, 4, 5], 8)
    c.logits, c.stride = flat, stride
    c.run().check()
