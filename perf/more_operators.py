"""Operators on a batch's rows around the attention, as timed cases in a plain form and as calls of libodma: the addition of a
block's output to the residual with the norms on both sides of it, the grouping of a batch's rows by low-rank adapter, the
adapters' products beside a shared projection, and log-probabilities of given tokens with entropy and best alternatives.
Sizes are those of the configurations, the benchmark and the tests of this repository (28 / 4 heads x 128: rows of 3584, a
projection of 4608 columns), or generic; draw() spreads over the ranges between and around them.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda"
ITEM_ROWS = 64                 # rows of an adapter item
NONE = -1                      # no adapter, no token, no row
ROW = {"f32": torch.float32, "bf16": torch.bfloat16}
ELEM = {"f32": 4, "bf16": 2}


def _norm(name, rows, *, dtype="bf16", residual="bf16", width=3584, post=True, gate="none", block_scale=1.0, residual_scale=1.0):
    return dict(name=name, kind="norm", rows=rows, dtype=dtype, residual=residual, width=width, post=post, gate=gate,
                block_scale=block_scale, residual_scale=residual_scale)


def _group(name, n, *, adapters=32, without=0.125, step=True, mid=512, hi=4096, lens_seed=1):
    return dict(name=name, kind="group", n=n, adapters=adapters, without=without, step=step, mid=mid, hi=hi, lens_seed=lens_seed)


def _adapt(name, n, *, dtype="bf16", adapters=32, without=0.0, step=True, mid=512, hi=4096, width=3584, cols="3584 512 512", rank=16,
           ragged=False, lens_seed=1):
    return dict(name=name, kind="adapt", n=n, dtype=dtype, adapters=adapters, without=without, step=step, mid=mid, hi=hi, width=width,
                cols=cols, rank=rank, ragged=ragged, lens_seed=lens_seed)


def _score(name, rows, *, dtype="bf16", vocab=128000, top=20, scale=1.0, masked=0.0, odd=False):
    return dict(name=name, kind="score", rows=rows, dtype=dtype, vocab=vocab, top=top, scale=scale, masked=masked, odd=odd)


def listed():
    return [
        # one user's next token: the residual stream between two blocks, latency alone
        _norm("norm_step_one", 1, post=False),
        # a decode step of the headline batch (256 requests): norms on both sides, a gate for every row and channel
        _norm("norm_step_b256", 256, gate="sigmoid"),
        # the benchmark's prompt mix, 16 x 4096 + 333 rows, residual in 32 bits, one learned scale for all rows
        _norm("norm_prompts_residual_f32", 16 * 4096 + 333, residual="f32", gate="row", residual_scale=0.5),
        # fp32 pools (8 heads x 65 channels), an odd number of rows
        _norm("norm_f32_narrow", 3001, dtype="f32", residual="f32", width=520, gate="value", block_scale=0.125),
        # the lists of a decode step: 256 requests over 32 adapters, one in eight without
        _group("group_step_b256", 256),
        # admission of 512 prompts with thousands of adapters loaded
        _group("group_prompts_b512", 512, adapters=4000, step=False, mid=128, hi=2048, lens_seed=6),
        # a decode step in which all 64 requests (config 2's batch) have an adapter of their own: the adapters' bytes
        _adapt("adapt_step_b64_all_different", 64, adapters=64, lens_seed=2),
        # prompts of twenty requests with eight adapters, beside the projection of queries, keys and values: the rows' bytes
        _adapt("adapt_prompts", 20, adapters=8, without=0.1, step=False, mid=2048, hi=16384, lens_seed=3),
        # fp32, larger adapters of different rank beside one projection, short prompts
        _adapt("adapt_f32_ragged", 24, dtype="f32", adapters=10, step=False, mid=64, hi=512, width=1000, cols="1024", rank=64, ragged=True,
               lens_seed=4),
        # one user's next token: a row of scores, its best twenty
        _score("score_step_one", 1),
        # a decode step of the headline batch, scores in 32 bits, temperature, some rows under a grammar
        _score("score_step_b256_f32", 256, dtype="f32", scale=1.25, masked=0.125),
        # log-probabilities of prompts: thousands of rows, a vocabulary of odd size whose rows lie densely
        _score("score_prompts_odd_vocab", 4096, vocab=50001, top=5, odd=True),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["norm", "norm", "group", "adapt", "adapt", "adapt", "score", "score", "score"])
    if kind == "norm":
        dtype = rng.choice(["bf16", "bf16", "f32"])
        c = _norm("", log_int(1, 65536), dtype=dtype, residual=rng.choice([dtype, "f32"]), width=8 * log_int(8, 2048), post=rng.random() < 0.5,
                  gate=rng.choice(["none", "row", "value", "sigmoid"]), block_scale=rng.choice([1.0, 0.25]),
                  residual_scale=rng.choice([1.0, 0.5]))
        budget = work(listed()[2])["bytes"]
        while work(c)["bytes"] > budget:
            c["rows"] = max(1, c["rows"] * 2 // 3)
    elif kind == "group":
        c = _group("", log_int(1, 1024), adapters=log_int(1, 20000), without=rng.choice([0.0, 0.125, 0.9]), step=rng.random() < 0.5,
                   mid=log_int(4, 256), hi=2048, lens_seed=rng.randrange(1 << 30))
        budget = work(listed()[5])["bytes"]
        while work(c)["bytes"] > budget:
            c["n"] = max(1, c["n"] * 2 // 3)
    elif kind == "adapt":
        parts = rng.choice([1, 1, 2, 3])
        c = _adapt("", log_int(1, 256), dtype=rng.choice(["bf16", "bf16", "f32"]), adapters=log_int(1, 128), without=rng.choice([0.0, 0.0, 0.3]),
                   step=rng.random() < 0.5, mid=log_int(4, 1024), hi=8192, width=8 * log_int(8, 1024),
                   cols=" ".join(str(16 * log_int(2, 256)) for _ in range(parts)), rank=8 * rng.choice([1, 1, 2, 2, 2, 3, 4, 8]), ragged=rng.random() < 0.4,
                   lens_seed=rng.randrange(1 << 30))
        budget = work(listed()[7])
        while work(c)["bytes"] > budget["bytes"] or work(c)["flops"] > 2 * budget["flops"]:
            if c["n"] > 1:
                c["n"] = max(1, c["n"] * 2 // 3)
            else:
                c["mid"], c["hi"] = max(1, c["mid"] // 2), max(1, c["hi"] // 2)
    else:
        c = _score("", log_int(1, 4096), dtype=rng.choice(["bf16", "f32"]), vocab=log_int(1000, 262144), top=rng.choice([0, 1, 5, 20, 64]),
                   scale=rng.choice([1.0, 1.0, 1.4]), masked=rng.choice([0.0, 0.0, 0.25, 1.0]), odd=rng.random() < 0.5)
        c["top"] = min(c["top"], c["vocab"])
        budget = work(listed()[11])["bytes"]
        while work(c)["bytes"] > budget:
            c["rows"] = max(1, c["rows"] * 2 // 3)
    del c["name"]
    return c


def _batch(case):
    """What a batch brings (host): every request's adapter, or NONE, and its rows."""
    rng = np.random.default_rng(case["lens_seed"])
    n = case["n"]
    if case["kind"] == "adapt" and case["step"] and case["adapters"] >= n:
        adapter = rng.permutation(case["adapters"])[:n]                 # as many as there are requests: each its own
    else:
        adapter = np.minimum(rng.geometric(min(1.0, 8.0 / case["adapters"]), n) - 1, case["adapters"] - 1)   # a few are popular
    adapter = np.where((rng.random(n) < case["without"]) & (np.arange(n) > 0), NONE, adapter).astype(np.int64)
    rows = np.clip(np.rint(np.exp(np.log(case["mid"]) + 0.8 * rng.standard_normal(n))), 1, case["hi"]).astype(np.int64)
    return adapter, np.ones(n, np.int64) if case["step"] else rows


def _cols(case):
    """The columns of the projections beside which the adapters stand, of each of them."""
    return [int(c) for c in case["cols"].split()]


def _ranks(case):
    """Every adapter's rank (host)."""
    if not case["ragged"]:
        return np.full(case["adapters"], case["rank"], np.int64)
    rng = np.random.default_rng(case["lens_seed"] + 1)
    return 8 * rng.integers(1, case["rank"] // 8 + 1, case["adapters"])


def _items(case):
    return int(_batch(case)[1].sum()) // ITEM_ROWS + min(case["n"], case["adapters"])


def work(case):
    if case["kind"] == "norm":
        e, f, r, w = ELEM[case["dtype"]], ELEM[case["residual"]], case["rows"], case["width"]
        gates = {"none": 0, "row": 1}.get(case["gate"], r)
        return {"bytes": r * w * (2 * e + 2 * f) + (gates + 1 + case["post"]) * w * e, "flops": r * w * 8}
    if case["kind"] == "score":
        r = case["rows"]
        return {"bytes": r * case["vocab"] * ELEM[case["dtype"]] + r * (4 + 12 + 8 * case["top"]), "flops": r * case["vocab"] * 6}
    adapter, rows = _batch(case)
    if case["kind"] == "group":
        return {"bytes": case["n"] * (4 + (0 if case["step"] else 8)) + int(rows.sum()) * 4 + _items(case) * 16, "flops": 0}
    e, rank = ELEM[case["dtype"]], _ranks(case)
    parts, cols, width = len(_cols(case)), sum(_cols(case)), case["width"]
    has = adapter >= 0
    there = rows[has]
    weights = int(rank[np.unique(adapter[has])].sum()) * (parts * width + cols) * e
    return {"bytes": int(there.sum()) * (width + 2 * cols) * e + weights,
            "flops": int((there * rank[adapter[has]]).sum()) * 2 * (parts * width + cols)}


# ---- what a program has in hand -------------------------------------------------------------------------------------------

def _handle(s, dtype, n):
    """The pool handle that a serving program keeps (its pools are not touched here)."""
    from paper_2512_09427_amd import binding as B
    kv = B.F32 if dtype == "f32" else B.BF16
    pool = torch.zeros(64 * 32, dtype=ROW[dtype], device=DEV)
    s["B"] = B
    s["pool"] = B.Pool(*B.make_config(n_layers=1, n_q_heads=1, n_kv_heads=1, head_dim=32, kv_dtype=kv, out_dtype=kv, main_tokens=32,
                                      safety_tokens=32, large_cap=16, boundaries=(16,), quantiles=((1, 2),), max_requests=n,
                                      k_pool=pool, v_pool=pool.clone()))


def _dev(a, dtype):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV).to(dtype)


def _prepare_norm(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    rows, w, typ, wide = case["rows"], case["width"], ROW[case["dtype"]], ROW[case["residual"]]

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=DEV)

    # a residual stream has a few channels that are far larger than the others, and rows of different size
    size = torch.where(torch.rand(w, generator=gen, device=DEV) < 0.004, 40.0, 1.0)
    s = dict(kind="norm", case=case, eps=1e-6, block=(normal(rows, w) * (0.2 + torch.rand(rows, 1, generator=gen, device=DEV))).to(typ),
             residual=(normal(rows, w) * size).to(wide), next_weight=(1 + 0.2 * normal(w)).to(typ),
             block_weight=(0.5 + 0.2 * normal(w)).to(typ) if case["post"] else None)
    s["gate"] = {"none": lambda: None, "row": lambda: (0.1 + 0.05 * normal(1, w)).to(typ)}.get(case["gate"], lambda: normal(rows, w).to(typ))()
    s["residual_out"], s["x_out"] = torch.empty(rows, w, dtype=wide, device=DEV), torch.empty(rows, w, dtype=typ, device=DEV)
    if own:
        _handle(s, case["dtype"], 1)
        B = s["B"]
        s["how"] = B.make_add_norm(width=w, block_weight=s["block_weight"], next_weight=s["next_weight"], gate=s["gate"],
                                   gate_kind={"none": B.GATE_NONE, "sigmoid": B.GATE_SIGMOID}.get(case["gate"], B.GATE_VALUE),
                                   gate_stride=0 if case["gate"] in ("none", "row") else w, eps=s["eps"],
                                   block_scale=case["block_scale"], residual_scale=case["residual_scale"],
                                   residual_dtype=B.F32 if case["residual"] == "f32" else B.BF16)
    return s


def _lists(adapter, rows, adapters, n_items):
    """Rows by adapter (host): their order, and items of up to ITEM_ROWS of them, adapter after adapter."""
    start = np.cumsum(rows) - rows
    by = [r for a in range(adapters) for r in np.flatnonzero(adapter == a)]
    order, items = np.full(int(rows.sum()), NONE, np.int64), np.zeros((n_items, 4), np.int64)
    items[:, 0] = NONE
    at, seen, i = 0, 0, 0
    while i < len(by):
        a, first = adapter[by[i]], at
        while i < len(by) and adapter[by[i]] == a:
            order[at:at + rows[by[i]]] = start[by[i]] + np.arange(rows[by[i]])
            at += rows[by[i]]
            i += 1
        for j in range(0, at - first, ITEM_ROWS):
            items[first // ITEM_ROWS + seen + j // ITEM_ROWS] = a, first + j, min(ITEM_ROWS, at - first - j), 0
        seen += 1
    return order, items


def _prepare_group(case, seed):
    # the batch's shape is the case's; which adapters it has is the seed's
    adapter, rows = _batch(case)
    names = np.random.default_rng(seed).permutation(case["adapters"])
    adapter = np.where(adapter >= 0, names[np.maximum(adapter, 0)], NONE)
    total = int(rows.sum())
    s = dict(kind="group", case=case, n=case["n"], adapters=case["adapters"], adapter=_dev(adapter, torch.int32), max_rows=total,
             row_start=None if case["step"] else _dev(np.concatenate([[0], np.cumsum(rows)]), torch.int64), max_items=_items(case))
    s["row_order"] = torch.empty(total, dtype=torch.int32, device=DEV)
    s["items"] = torch.empty(s["max_items"], 4, dtype=torch.int32, device=DEV)
    if own:
        _handle(s, "bf16", case["n"])
    return s


def _prepare_adapt(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    adapter, rows = _batch(case)
    names = np.random.default_rng(seed).permutation(case["adapters"])
    adapter = np.where(adapter >= 0, names[np.maximum(adapter, 0)], NONE)
    rank = np.empty(case["adapters"], np.int64)
    rank[names] = _ranks(case)
    total, typ, parts, cols = int(rows.sum()), ROW[case["dtype"]], len(_cols(case)), sum(_cols(case))
    order, items = _lists(adapter, rows, case["adapters"], _items(case))

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=DEV)

    # weights of adapters below the largest rank stand in arrays that were made for it; the rest is zeros
    held = torch.arange(case["rank"], device=DEV) < _dev(rank, torch.int64)[:, None]
    down = (normal(case["adapters"], parts, case["rank"], case["width"]) / math.sqrt(case["width"])).to(typ)
    down *= held[:, None, :, None]
    up = (0.5 * normal(case["adapters"], cols, case["rank"])).to(typ)
    up *= held[:, None]
    s = dict(kind="adapt", case=case, down=down, up=up, scale=0.25 + torch.rand(case["adapters"], generator=gen, device=DEV),
             ranks=_dev(rank, torch.int32), items=_dev(items, torch.int32), row_order=_dev(order, torch.int32),
             total=total, max_items=len(items),
             x=normal(total, case["width"]).to(typ), base=normal(total, cols).to(typ))
    s["y"] = s["base"].clone()                       # rows without an adapter keep the projection's values
    if own:
        _handle(s, case["dtype"], case["n"])
        s["adapters"] = s["B"].make_adapters(down=s["down"], up=s["up"], n_adapters=case["adapters"], rank=case["rank"], width=case["width"],
                                             part_cols=_cols(case), scale=s["scale"], ranks=s["ranks"] if case["ragged"] else None)
        s["scratch"] = torch.empty(s["pool"].odma_adapt_scratch_bytes(s["adapters"], s["max_items"]), dtype=torch.uint8, device=DEV)
    return s


def _prepare_score(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    rows, vocab, typ = case["rows"], case["vocab"], ROW[case["dtype"]]
    # rows of an odd vocabulary lie densely, others as wide as the next multiple of 64
    stride = vocab + (1 - vocab % 2 if case["odd"] else -vocab % 64)
    logits = torch.randn(rows, stride, generator=gen, device=DEV)
    logits *= 1.0 + 2.0 * torch.rand(rows, 1, generator=gen, device=DEV)
    # a few words that fit
    at = torch.randint(0, vocab, (rows, 4), generator=gen, device=DEV)
    logits.scatter_add_(1, at, 12.0 * torch.rand(rows, 4, generator=gen, device=DEV))
    # under a grammar: most words are switched off, in some rows all but three
    for r in range(int(rows * case["masked"] + 0.5) if rows <= 256 else 0):
        keep = torch.rand(stride, generator=gen, device=DEV) < 0.2
        if r % 4 == 3:
            keep[:] = False
        keep[at[r, :3]] = True
        logits[r].masked_fill_(~keep, -math.inf)
    logits = logits.to(typ)
    # the tokens that were drawn, or came next in the text
    noise = -torch.log(-torch.log(torch.rand(rows, 1024, generator=gen, device=DEV).clamp(1e-30, 1 - 1e-7)))
    pick = torch.randint(0, vocab, (rows, 1024), generator=gen, device=DEV)
    tokens = pick.gather(1, (logits.gather(1, pick).float() + noise).argmax(1, keepdim=True))[:, 0]
    tokens = torch.where(torch.rand(rows, generator=gen, device=DEV) < 0.5, at[:, 0], tokens)
    s = dict(kind="score", case=case, logits=logits, stride=stride, tokens=tokens.int())
    s["logprob"], s["entropy"] = torch.empty(2, rows, device=DEV).unbind(0)
    s["rank"] = torch.empty(rows, dtype=torch.int32, device=DEV)
    s["top_id"] = torch.empty(rows, case["top"], dtype=torch.int32, device=DEV)
    s["top_logprob"] = torch.empty(rows, case["top"], device=DEV)
    if own:
        _handle(s, case["dtype"], 1)
        s["scratch"] = torch.empty(s["pool"].odma_score_scratch_bytes(rows, vocab, case["top"]), dtype=torch.uint8, device=DEV)
    return s


def prepare(case, seed):
    return {"norm": _prepare_norm, "group": _prepare_group, "adapt": _prepare_adapt, "score": _prepare_score}[case["kind"]](case, seed)


# ---- plain forms -----------------------------------------------------------------------------------------------------------

def _plain_norm(s):
    c = s["case"]
    b = s["block"].float()
    if s["block_weight"] is not None:
        b = b * torch.rsqrt(b.square().mean(-1, keepdim=True) + s["eps"]) * s["block_weight"].float()
    if s["gate"] is not None:
        g = s["gate"].float()
        b = b * (torch.sigmoid(g) if c["gate"] == "sigmoid" else g)
    r = c["residual_scale"] * s["residual"].float() + c["block_scale"] * b
    s["residual_out"].copy_(r)
    s["x_out"].copy_(r * torch.rsqrt(r.square().mean(-1, keepdim=True) + s["eps"]) * s["next_weight"].float())
    return s["residual_out"], s["x_out"]


def _plain_group(s):
    n, adapters, adapter = s["n"], s["adapters"], s["adapter"].long()
    rows = torch.ones_like(adapter) if s["row_start"] is None else s["row_start"].diff()
    start = rows.cumsum(0) - rows
    group = torch.where((adapter >= 0) & (adapter < adapters), adapter, adapters)   # behind the others: without one
    group, by = torch.sort(group, stable=True)
    placed = torch.where(group < adapters, rows[by], 0)
    ends = placed.cumsum(0)
    at = torch.arange(s["max_rows"], device=DEV)
    r = torch.searchsorted(ends, at, right=True).clamp(max=n - 1)
    order = torch.where(at < ends[-1], start[by][r] + at - (ends - placed)[r], NONE)
    count = torch.zeros(adapters + 1, dtype=torch.int64, device=DEV).scatter_add_(0, group, placed)[:adapters]
    first = count.cumsum(0) - count
    slot = first // ITEM_ROWS + (count > 0).long().cumsum(0) - (count > 0).long()
    ends = torch.where(count > 0, slot + (count + ITEM_ROWS - 1) // ITEM_ROWS, 0).cummax(0).values
    i = torch.arange(s["max_items"], device=DEV)
    a = torch.searchsorted(ends, i, right=True).clamp(max=adapters - 1)
    j = (i - slot[a]) * ITEM_ROWS
    there = (i >= slot[a]) & (j < count[a])
    item = torch.stack([a, first[a] + j, (count[a] - j).clamp(max=ITEM_ROWS), torch.zeros_like(a)], 1)
    empty = torch.tensor([NONE, 0, 0, 0], device=DEV)
    return order.int(), torch.where(there[:, None], item, empty).int()


def _plain_adapt(s):
    items, width = s["items"].long(), s["x"].shape[1]
    there = items[:, 2] > 0
    j = torch.arange(ITEM_ROWS, device=DEV)[None]
    held = j < items[:, 2:3]
    row = s["row_order"].long()[torch.where(held, items[:, 1:2] + j, 0)]
    row = torch.where(held, row, s["total"])
    a = torch.where(there, items[:, 0], 0)
    down, up = s["down"][a].float(), s["up"][a].float()                        # [item][part][rank][width], [item][cols][rank]
    parts, rank = down.shape[1:3]
    x = s["x"].float()[row.clamp(max=s["total"] - 1)]
    h = torch.bmm(x, down.view(-1, parts * rank, width).transpose(1, 2).contiguous()).view(-1, ITEM_ROWS, parts, rank)
    h = h * s["scale"][a][:, None, None, None]
    y = torch.empty(s["total"] + 1, s["base"].shape[1], device=DEV)            # (the last row takes what belongs to none)
    y[:-1] = s["base"].float()
    ends = np.cumsum([0] + _cols(s["case"])).tolist()
    parted = [torch.bmm(h[:, :, p].contiguous(), up[:, ends[p]:ends[p + 1]].transpose(1, 2).contiguous()) for p in range(parts)]
    at = row.reshape(-1)
    y[at] = y[at] + torch.cat(parted, 2).reshape(at.shape[0], -1)
    s["y"].copy_(y[:-1])
    return s["y"]


def _plain_score(s):
    c = s["case"]
    vocab, top = c["vocab"], c["top"]
    raw = s["logits"][:, :vocab].float() + 0.0                                  # (-0 and 0 are the same score)
    token = s["tokens"].long()[:, None]
    x = raw * c["scale"]
    m = x.amax(-1, keepdim=True)
    d = x - m
    e = torch.exp(d)
    z = e.sum(-1, keepdim=True)
    logz = torch.log(z)
    entropy = (logz - torch.where(e > 0, e * d, 0.0).sum(-1, keepdim=True) / z)[:, 0]
    logprob = (d.gather(1, token) - logz)[:, 0]
    rank = (raw > raw.gather(1, token)).sum(-1).int()
    # the largest, ties by index: one whole number for both, the scores' bits in an order that whole numbers have too
    bits = raw.view(torch.int32)
    key = torch.where(bits < 0, bits ^ 0x7fffffff, bits).long() * (1 << 32) + ((1 << 31) - torch.arange(vocab, device=DEV))
    at = torch.topk(key, top, dim=1).indices
    off = raw.gather(1, at) == -math.inf
    return logprob, rank, entropy, torch.where(off, NONE, at).int(), d.gather(1, at) - logz


# ---- one pass ----------------------------------------------------------------------------------------------------------------

def _run_norm(s):
    if not own:
        return _plain_norm(s)
    w = s["case"]["width"]
    s["pool"].odma_add_norm(s["case"]["rows"], s["how"], s["block"], w, s["residual"], w, None, s["residual_out"], s["x_out"])
    return s["residual_out"], s["x_out"]


def _run_group(s):
    if not own:
        return _plain_group(s)
    s["pool"].odma_group_adapters(s["n"], s["adapter"], s["adapters"], s["row_start"], s["max_rows"], s["row_order"], s["max_items"], s["items"])
    return s["row_order"], s["items"]


def _run_adapt(s):
    if not own:
        return _plain_adapt(s)
    x, cols = s["x"], s["base"].shape[1]
    s["pool"].odma_adapt_rows(s["total"], s["adapters"], s["max_items"], s["items"], s["row_order"], x, x.shape[1], s["base"], cols, s["y"], cols,
                              s["scratch"])
    return s["y"]


def _run_score(s):
    if not own:
        return _plain_score(s)
    c, B = s["case"], s["B"]
    top = c["top"] > 0
    s["pool"].odma_score_tokens(c["rows"], s["logits"], s["stride"], B.F32 if c["dtype"] == "f32" else B.BF16, c["vocab"], c["scale"], s["tokens"],
                                None, c["top"], s["logprob"], s["rank"], s["entropy"], s["top_id"] if top else None,
                                s["top_logprob"] if top else None, s["scratch"])
    return s["logprob"], s["rank"], s["entropy"], s["top_id"], s["top_logprob"]


def run(state):
    return {"norm": _run_norm, "group": _run_group, "adapt": _run_adapt, "score": _run_score}[state["kind"]](state)


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------------------

def _exact_norm(case, s):
    def normed(x, weight):
        return x / ((x * x).sum(-1, keepdim=True) / case["width"] + s["eps"]).sqrt() * weight.double()

    residual = torch.empty(case["rows"], case["width"], dtype=torch.float64, device=DEV)
    x = torch.empty_like(residual)
    for at in range(0, case["rows"], 8192):
        some = slice(at, at + 8192)
        b = s["block"][some].double()
        if case["post"]:
            b = normed(b, s["block_weight"])
        if case["gate"] != "none":
            g = s["gate"].double() if case["gate"] == "row" else s["gate"][some].double()
            b = b / (1 + (-g).exp()) if case["gate"] == "sigmoid" else b * g
        residual[some] = s["residual"][some].double() * case["residual_scale"] + b * case["block_scale"]
        x[some] = normed(residual[some], s["next_weight"])
    return residual, x


def _exact_adapt(case, s):
    y = s["base"].double()
    for adapter, first, count, _ in s["items"].tolist():
        if count:
            row = s["row_order"][first:first + count].long()
            x, at = s["x"][row].double(), 0
            for p, cols in enumerate(_cols(case)):
                h = x @ s["down"][adapter, p].double().T.contiguous()
                y[row, at:at + cols] += (h @ s["up"][adapter, at:at + cols].double().T.contiguous()) * s["scale"][adapter].double()
                at += cols
    return y


def _exact_score(case, s):
    logprob, entropy, best = [], [], []
    for at in range(0, case["rows"], 64):
        x = s["logits"][at:at + 64, :case["vocab"]].double()
        lp = torch.log_softmax(x * case["scale"], -1)
        logprob.append(lp.gather(1, s["tokens"][at:at + 64].long()[:, None])[:, 0])
        entropy.append(-torch.xlogy(lp.exp(), lp.exp()).sum(-1))
        best.append(lp.sort(-1, descending=True).values[:, :case["top"]])
    return torch.cat(logprob), None, torch.cat(entropy), None, torch.cat(best)


def exact(case, seed):
    if case["kind"] == "group":
        return None
    return {"norm": _exact_norm, "adapt": _exact_adapt, "score": _exact_score}[case["kind"]](case, prepare(case, seed))
