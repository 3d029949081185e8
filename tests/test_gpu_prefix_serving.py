"""The calls together, as a serving program makes them: two system prompts fill shared slabs, requests behind them bring their own
prompts (tables, rows with norms and rotations into paged or contiguous slabs, prompt attention over the tables), then decode steps
whose tables, rows and attention run in one captured graph while lengths grow on the GPU.  Attention is checked in 64 bits
against the K and V that the pool holds, read back, and the rows against their formula; queries as the rows call left them."""
import math

import numpy as np
import pytest
import torch

from paper_2512_09427_amd import binding as B

DEV = "cuda"
pytestmark = pytest.mark.gpu
HQ, HKV, D, EPS = 14, 2, 128, 1e-6
PREFIX = [530, 100]                                             # 528 and 96 tokens are shared
GROUPS = [(0, 3), (3, 5)]                                       # and request 5 has no prefix
OWN = [40, 7, 100, 33, 16, 61]                                  # tokens behind the prefix


class Server:
    def __init__(self, kvd, paged):
        self.kvd, self.paged, self.n = kvd, paged, len(OWN)
        gen = torch.Generator(device=DEV).manual_seed(4)
        self.gen = gen
        self.tokens = 4096
        raw = torch.uint8 if kvd == "fp8" else torch.bfloat16
        self.k_pool, self.v_pool = (torch.full((HKV * (self.tokens + 256) * D,), 0x7f if kvd == "fp8" else float("nan"), dtype=raw, device=DEV)
                                    for _ in range(2))
        args = dict(n_layers=1, n_q_heads=HQ, n_kv_heads=HKV, head_dim=D, kv_dtype=B.FP8 if kvd == "fp8" else B.BF16, out_dtype=B.F32,
                    main_tokens=self.tokens, safety_tokens=256, large_cap=256, boundaries=(256,), quantiles=((1, 2),), max_requests=16)
        self.scale = 2.0 ** -6 if kvd == "fp8" else 1.0
        if kvd == "fp8":
            args.update(k_scale=self.scale, v_scale=self.scale)
        ws = torch.empty(B.odma_workspace_bytes(B.make_config(**args)[0]), dtype=torch.uint8, device=DEV)
        self.pool = B.Pool(*B.make_config(**args, k_pool=self.k_pool, v_pool=self.v_pool, workspace=ws))
        rc, _, off, _, _ = self.pool.odma_assign(np.arange(self.n), np.full(self.n, 200))
        assert rc == 0
        self.off = torch.tensor(off, device=DEV)
        self.pre = torch.tensor([2048, 2592], dtype=torch.int64, device=DEV)     # (prefix slabs: the rest of the arena is the caller's)
        self.start = torch.tensor([0, 3, 5], dtype=torch.int32, device=DEV)
        self.plen = torch.tensor(PREFIX, dtype=torch.int32, device=DEV)
        self.wq, self.wk = ((1 + 0.2 * torch.randn(D, generator=gen, device=DEV)).bfloat16() for _ in range(2))
        self.inv_freq = (10000.0 ** (-torch.arange(0, D, 2, device=DEV) / D)).float()
        self.prep = B.make_qk_prep(q_weight=self.wq, k_weight=self.wk, eps=EPS, rot_dim=D, inv_freq=self.inv_freq)

    def project(self, rows):
        return torch.randn(rows, (HQ + 2 * HKV) * D, generator=self.gen, device=DEV).bfloat16()

    def rows(self, qkv, slot, pos, q_out):
        n = qkv.shape[0]
        self.pool.odma_append_qkv(0, n, self.prep, qkv, qkv.shape[1], qkv[:, HQ * D:], qkv.shape[1], qkv[:, (HQ + HKV) * D:], qkv.shape[1],
                                  slot, pos, q_out)

    def stored(self):
        """K and V of every token slot as numbers, and the slots of a request's tokens."""
        k = torch.empty(self.tokens + 256, HKV, D, dtype=self.k_pool.dtype, device=DEV)
        v = torch.empty_like(k)
        self.pool.odma_gather_kv(0, 0, self.tokens + 256, None, k, v)
        f8 = torch.float8_e4m3fn
        return [(x.view(f8).double() if self.kvd == "fp8" else x.double()) * self.scale for x in (k, v)]

    def slots_of(self, r, length):
        group = next((p for p, (a, b) in enumerate(GROUPS) if a <= r < b), None)
        shared = PREFIX[group] // 16 * 16 if group is not None else 0
        t = torch.arange(length, device=DEV)
        return torch.where(t < shared, int(self.pre[group]) + t if group is not None else t, int(self.off[r]) + t - shared)

    def attend(self, q, slots, k, v):
        kk, vv = (x[slots].repeat_interleave(HQ // HKV, 1) for x in (k, v))
        p = torch.softmax((kk * q.double()).sum(-1) / math.sqrt(D), 0)
        return (p[..., None] * vv).sum(0), (p[..., None] * vv.abs()).sum(0)

    def queries(self, qkv, pos):
        """What the rows call leaves of the queries, in 64 bits."""
        x = qkv[:, :HQ * D].double().view(-1, HQ, D)
        x = x * (x.square().mean(-1, keepdim=True) + EPS).rsqrt() * self.wq.double()
        angle = (pos.double()[:, None] * self.inv_freq.double())[:, None]
        a, b = x[..., :D // 2], x[..., D // 2:]
        return torch.cat([a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin()], -1)


def build(s, lengths, new, table, row_start, pos, slot):
    s.pool.odma_build_tables(s.n, lengths, new, s.off, 2, s.start, s.pre, s.plen, table, table.shape[1], pos.shape[0], row_start, pos, slot)


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("kvd", ["bf16", "fp8"])
def test_prompts_and_steps_behind_shared_prefixes(kvd, paged):
    s = Server(kvd, paged)
    i32, i64 = dict(dtype=torch.int32, device=DEV), dict(dtype=torch.int64, device=DEV)
    # the prefixes: rows like any others, straight into their slabs (their last tokens are not shared, and not read there)
    for p, length in enumerate(PREFIX):
        t = torch.arange(length, **i32)
        s.rows(s.project(length), t.long() + s.pre[p], t, torch.empty(length, HQ, D, dtype=torch.bfloat16, device=DEV))
    whole = [(PREFIX[0] // 16 * 16 if r < 3 else PREFIX[1] // 16 * 16 if r < 5 else 0) for r in range(s.n)]
    new = torch.tensor(OWN, **i32)
    lengths = torch.tensor([w + o for w, o in zip(whole, OWN)], **i32)
    total, spare, stride = sum(OWN), 11, 48
    table, row_start = torch.empty(s.n, stride, **i32), torch.empty(s.n + 1, **i64)
    pos, slot = torch.empty(total + spare, **i32), torch.empty(total + spare, **i64)
    build(s, lengths, new, table, row_start, pos, slot)
    qkv = s.project(total + spare)
    q = torch.full((total + spare, HQ, D), 7.0, dtype=torch.bfloat16, device=DEV)
    s.rows(qkv, slot, pos, q)
    assert (q[total:] == 7).all()                                # rows behind the last request's
    want = s.queries(qkv[:total], pos[:total])
    assert ((q[:total].double() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-5).all()
    out = torch.full((total + spare, HQ, D), float("nan"), device=DEV)
    s.pool.odma_prefill_attention(0, s.n, q, total + spare, row_start, new, None, lengths, table, stride, out)
    k, v = s.stored()
    for r in range(s.n):
        a, b = int(row_start[r]), int(row_start[r + 1])
        assert b - a == OWN[r]
        for j in range(a, b, 5):
            seen = int(pos[j]) + 1
            ref, size = s.attend(q[j], s.slots_of(r, seen), k, v)
            # (the weights of a prompt are bf16 numbers: 2^-8 of what they average, and fp8's scores a few 2^-8)
            assert ((out[j].double() - ref).abs() <= 2.0 ** -7 * size + 1e-6).all()
    assert torch.isnan(out[total:]).all()
    # decode: one token each, planned, prepared and attended to in a captured graph; request 1 is finished after two steps
    one, spos, sslot = torch.empty(s.n + 1, **i64), torch.empty(s.n, **i32), torch.empty(s.n, **i64)
    sqkv, sq = s.project(s.n), torch.zeros(s.n, HQ, D, dtype=torch.bfloat16, device=DEV)
    sout = torch.empty(s.n, HQ, D, device=DEV)

    def step():
        lengths.add_((lengths > 0).int())
        build(s, lengths, None, table, one, spos, sslot)
        s.rows(sqkv, sslot, spos, sq)
        s.pool.odma_decode_attention_shared(0, s.n, sq, 2, s.start, s.pre, s.plen, None if s.paged else s.off, lengths,
                                            table if s.paged else None, stride if s.paged else 0, sout)

    side = torch.cuda.Stream()
    kept = lengths.clone()
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    lengths.copy_(kept)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    lengths.copy_(kept)
    at = kept.tolist()
    for i in range(6):
        sqkv.copy_(s.project(s.n))
        sout.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        at = [x + (x > 0) for x in at]
        assert lengths.tolist() == at
        k, v = s.stored()
        live = [r for r in range(s.n) if at[r] > 0]
        assert int(one[s.n]) == len(live)
        for j, r in enumerate(live):                             # rows are dense: an empty place has none
            assert int(spos[j]) == at[r] - 1 and int(sslot[j]) == int(s.slots_of(r, at[r])[-1])
        dense = len(live) == s.n
        for r in range(s.n):
            if at[r] == 0:
                assert (sout[r] == 0).all()
                continue
            ref, size = s.attend(sq[r], s.slots_of(r, at[r]), k, v)
            assert ((sout[r].double() - ref).abs() <= 2.0 ** -14 * size + 1e-6).all(), (i, r)
        if dense and i == 2:
            lengths[5] = 0                                        # the last place empties: the other rows stay where they are
            at[5] = 0


def test_slabs_past_32_bits():
    """The same batch in slabs at the beginning of a pool and behind 4 GiB of one head's rows: the same results, bit for bit."""
    n, own, shared = 3, [40, 1, 77], 160
    tokens = (1 << 24) + 65536
    pools = [torch.zeros((tokens + 256) * D, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    args = dict(n_layers=1, n_q_heads=4, n_kv_heads=1, head_dim=D, kv_dtype=B.BF16, out_dtype=B.F32, main_tokens=tokens, safety_tokens=256,
                large_cap=256, boundaries=(256,), quantiles=((1, 2),), max_requests=4)
    ws = torch.empty(B.odma_workspace_bytes(B.make_config(**args)[0]), dtype=torch.uint8, device=DEV)
    pool = B.Pool(*B.make_config(**args, k_pool=pools[0], v_pool=pools[1], workspace=ws))
    gen = torch.Generator(device=DEV).manual_seed(9)
    i32, i64 = dict(dtype=torch.int32, device=DEV), dict(dtype=torch.int64, device=DEV)
    start, plen = torch.tensor([0, 3], **i32), torch.tensor([shared + 5], **i32)
    lengths, new = torch.tensor([shared + o for o in own], **i32), torch.tensor(own, **i32)
    total = sum(own)
    qkv = torch.randn(shared + total, 6 * D, generator=gen, device=DEV).bfloat16()
    prep = B.make_qk_prep(rot_dim=D, inv_freq=(10000.0 ** (-torch.arange(0, D, 2, device=DEV) / D)).float())
    results = []
    for base in (0, (1 << 24) + 4096):
        pre = torch.tensor([base + 512], **i64)
        off = torch.tensor([base, base + 1024, base + 2048], **i64)
        pos, slot = torch.empty(total, **i32), torch.empty(total, **i64)
        table = torch.empty(n, 16, **i32)
        pool.odma_build_tables(n, lengths, new, off, 1, start, pre, plen, table, 16, total, None, pos, slot)
        assert slot.tolist() == [base + o + j for o, c in zip((0, 1024, 2048), own) for j in range(c)]
        t = torch.arange(shared, **i32)
        q = torch.empty(shared + total, 4, D, dtype=torch.bfloat16, device=DEV)
        for rows, s, p in ((slice(0, shared), pre + t, t), (slice(shared, None), slot, pos)):
            x = qkv[rows]
            pool.odma_append_qkv(0, x.shape[0], prep, x, 6 * D, x[:, 4 * D:], 6 * D, x[:, 5 * D:], 6 * D, s, p, q[rows])
        for bt in (None, table):
            out = torch.empty(n, 4, D, device=DEV)
            pool.odma_decode_attention_shared(0, n, q[:n].contiguous(), 1, start, pre, plen, off, lengths, bt, 0 if bt is None else 16, out)
            results.append(out)
    for other in results[1:]:
        assert torch.equal(other, results[0])
    assert torch.isfinite(results[0]).all() and results[0].abs().max() > 0


@pytest.mark.parametrize("by_place", [False, True])
@pytest.mark.parametrize("kvd", ["bf16", "fp8"])
def test_places_that_empty_in_the_middle(kvd, by_place):
    """A captured loop of decode steps in which requests end in the middle of the batch and a place is filled again.  Rows are dense: behind
    an empty place they move up, and row_start leads from requests to rows.  Either attention's queries are gathered by it, or slots
    and positions are laid out by place, with ODMA_SLOT_NONE for the empty ones."""
    s = Server(kvd, False)
    n = s.n
    i32, i64 = dict(dtype=torch.int32, device=DEV), dict(dtype=torch.int64, device=DEV)
    for p, length in enumerate(PREFIX):
        t = torch.arange(length, **i32)
        s.rows(s.project(length), t.long() + s.pre[p], t, torch.empty(length, HQ, D, dtype=torch.bfloat16, device=DEV))
    whole = [(PREFIX[0] // 16 * 16 if r < 3 else PREFIX[1] // 16 * 16 if r < 5 else 0) for r in range(n)]
    own, lengths = torch.tensor(OWN, **i32), torch.tensor([w + o for w, o in zip(whole, OWN)], **i32)
    start, pos, slot = torch.empty(n + 1, **i64), torch.empty(sum(OWN), **i32), torch.empty(sum(OWN), **i64)
    table = torch.empty(n, 48, **i32)
    build(s, lengths, own, table, start, pos, slot)
    s.rows(s.project(sum(OWN)), slot, pos, torch.empty(sum(OWN), HQ, D, dtype=torch.bfloat16, device=DEV))
    pos, slot = torch.empty(n, **i32), torch.empty(n, **i64)
    qkv, q, out = s.project(n), torch.zeros(n, HQ, D, dtype=torch.bfloat16, device=DEV), torch.empty(n, HQ, D, device=DEV)
    place_pos, place_slot, asked = torch.empty_like(pos), torch.empty_like(slot), torch.empty_like(q)

    def step():
        lengths.add_((lengths > 0).int())
        build(s, lengths, None, table, start, pos, slot)
        row = start[:n].clamp(max=n - 1)
        if by_place:
            place_slot.copy_(torch.where(start[1:] > start[:n], slot[row], B.SLOT_NONE))
            place_pos.copy_(pos[row])
            s.rows(qkv, place_slot, place_pos, q)
            asked.copy_(q)
        else:
            s.rows(qkv, slot, pos, q)
            asked.copy_(q[row])
        s.pool.odma_decode_attention_shared(0, n, asked, 2, s.start, s.pre, s.plen, s.off, lengths, None, 0, out)

    kept = lengths.clone()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    lengths.copy_(kept)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    lengths.copy_(kept)
    at = kept.tolist()
    for i in range(7):
        if i in (2, 3):                                           # requests 1 and 4 end, one step apart
            at[(1, 4)[i - 2]] = 0
        if i == 5:                                                # another one in place 1, its tokens are there already
            at[1] = whole[1] + 9
        lengths.copy_(torch.tensor(at, **i32))
        qkv.copy_(s.project(n))
        q.fill_(float("nan"))
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        at = [x + (x > 0) for x in at]
        assert lengths.tolist() == at
        k, v = s.stored()
        live = [r for r in range(n) if at[r] > 0]
        assert int(start[n]) == len(live) == n - [0, 0, 1, 2, 2, 1, 1][i]
        for r in range(n):
            if at[r] == 0:
                assert (out[r] == 0).all()
                continue
            row = r if by_place else live.index(r)
            here = s.slots_of(r, at[r])
            assert int((place_slot if by_place else slot)[row]) == int(here[-1])
            want = s.queries(qkv[row:row + 1], torch.tensor([at[r] - 1], device=DEV))[0]
            assert ((q[row].double() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-5).all()
            moved = qkv[row, (HQ + HKV) * D:].double().view(HKV, D)       # (values go into the pool as they are; E4M3: half a step)
            assert ((v[here[-1]] - moved).abs() <= (2.0 ** -4 * moved.abs() + s.scale * 2.0 ** -10 if kvd == "fp8" else 0.0)).all()
            ref, size = s.attend(q[row], here, k, v)
            assert ((out[r].double() - ref).abs() <= 2.0 ** -14 * size + 1e-6).all(), (i, r)
