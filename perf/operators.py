"""Serving operators around the KV pools, as timed cases in a plain form and as calls of libodma: the tables of a batch
(block tables, row starts, token slots, with prefixes that several requests share), the rows between the projections
and the attention (norms of queries and keys for each head, rotary positions on one or several axes, the append into the
pools), and decode attention over a batch that shares long prefixes.  Sizes are those of the configurations, the
benchmark and the tests of this repository; draw() spreads over the ranges between and around them.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda"
BLOCK = 16
FP8_SCALE = 2.0 ** -6          # stored E4M3 value = real value / FP8_SCALE
INPUT = {"f32": torch.float32, "bf16": torch.bfloat16, "fp8": torch.bfloat16}
STORE = {"f32": torch.float32, "bf16": torch.bfloat16, "fp8": torch.float8_e4m3fn}
ELEM = {"f32": 4, "bf16": 2, "fp8": 1}
SLOT_NONE, SLOT_SHARED = -1, -2


def _tables(name, n, *, new=0, mid=512, hi=4096, prefixes=0, shared=0, lens_seed=1):
    return dict(name=name, kind="tables", n=n, new=new, mid=mid, hi=hi, prefixes=prefixes, shared=shared, lens_seed=lens_seed)


def _rows(name, rows, *, dtype="bf16", hq=28, hkv=4, d=128, norm=True, rot=128, adjacent=False, axes=1, run=0, far=32768):
    return dict(name=name, kind="rows", rows=rows, dtype=dtype, hq=hq, hkv=hkv, d=d, norm=norm, rot=rot, adjacent=adjacent,
                axes=axes, run=run, far=far)


def _shared(name, n, *, dtype="bf16", hq=28, hkv=4, d=128, prefixes=1, shared=4096, mid=512, hi=4096, paged=False, out="bf16",
            lens_seed=1):
    return dict(name=name, kind="shared", n=n, dtype=dtype, hq=hq, hkv=hkv, d=d, prefixes=prefixes, shared=shared, mid=mid,
                hi=hi, paged=paged, out=out, lens_seed=lens_seed)


def listed():
    return [
        # the tables of one decode step of an ordinary batch (config 2's lengths): latency alone counts
        _tables("tables_step_b64", 64, new=1, lens_seed=2),
        # admission of 256 prompts behind four system prompts: a slot for each of their rows
        _tables("tables_prompts_b256", 256, mid=1024, hi=16384, prefixes=4, shared=1024, lens_seed=6),
        # a step of the largest batch there is, contexts up to the longest request of config 5
        _tables("tables_step_b1024_long", 1024, new=1, mid=2048, hi=65536, lens_seed=5),
        # one user's next token: norms, rotation and append of a single row
        _rows("rows_step_one", 1),
        # a decode step of the headline batch (config 3): 256 rows, each somewhere else in the pool
        _rows("rows_step_b256", 256),
        # the benchmark's prompt mix, 16 x 4096 + 333 rows
        _rows("rows_prompts", 16 * 4096 + 333, run=4096),
        # images and video in a byte-wide pool: positions on three axes, an odd number of rows
        _rows("rows_three_axes_fp8", 20011, dtype="fp8", axes=3, run=1777),
        # fp32 pools (config 1's head size), half of each head rotated, neighbouring channels as pairs, no norm
        _rows("rows_f32_partial", 3001, dtype="f32", hq=8, hkv=2, d=64, norm=False, rot=32, adjacent=True, run=333),
        # a few requests behind one system prompt of odd length: latency
        _shared("shared_b8", 8, shared=1000, mid=128, hi=1024),
        # an ordinary batch (config 2's lengths) behind a long prompt with documents in it
        _shared("shared_b64", 64, shared=4096, lens_seed=2),
        # many short answers to questions about one very long text: the prefix is a matrix product
        _shared("shared_b256_long", 256, shared=16384, mid=256, hi=2048, lens_seed=3),
        # byte-wide paged pools, four prompts of different length, one request in eight without any
        _shared("shared_b128_fp8_paged", 128, dtype="fp8", prefixes=4, shared=2048, mid=384, hi=4096, paged=True, lens_seed=4),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["tables", "rows", "rows", "shared", "shared"])
    if kind == "tables":
        c = _tables("", log_int(1, 1024), new=rng.choice([0, 1, 1, 5]), mid=log_int(16, 2048), prefixes=rng.choice([0, 0, 1, 3, 8]),
                    shared=log_int(16, 4096), lens_seed=rng.randrange(1 << 30))
        c["hi"] = min(c["mid"] * log_int(2, 32), 65536)
        c["prefixes"] = min(c["prefixes"], c["n"])
        budget = work(listed()[2])["bytes"]
        while work(c)["bytes"] > budget:
            c["n"] = max(1, c["n"] * 2 // 3)
            c["prefixes"] = min(c["prefixes"], c["n"])
    elif kind == "rows":
        dtype, d = rng.choice([("bf16", 128), ("bf16", 128), ("bf16", 64), ("fp8", 128), ("fp8", 128), ("f32", 64), ("f32", 128),
                               ("bf16", 96), ("bf16", 256)])
        hkv = rng.choice([1, 2, 3, 4, 8])
        c = _rows("", log_int(1, 65536), dtype=dtype, d=d, hkv=hkv, hq=hkv * rng.randint(1, 8), norm=rng.random() < 0.6,
                  rot=rng.choice([d, d, d // 2, 24]), adjacent=rng.random() < 0.3, axes=rng.choice([1, 1, 3]),
                  run=rng.choice([0, log_int(3, 8192)]), far=rng.choice([4096, 32768, 1000000]))
        budget = work(listed()[5])["bytes"]
        while work(c)["bytes"] > budget:
            c["rows"] = max(1, c["rows"] * 2 // 3)
    else:
        dtype, d = rng.choice([("bf16", 128), ("bf16", 128), ("bf16", 64), ("fp8", 128)])
        hkv = rng.choice([1, 2, 3, 4, 8])
        c = _shared("", log_int(1, 256), dtype=dtype, d=d, hkv=hkv, hq=hkv * rng.randint(1, 8), prefixes=rng.choice([1, 1, 2, 5]),
                    shared=log_int(16, 32768), mid=log_int(16, 1024), paged=rng.random() < 0.4,
                    out=rng.choice(["bf16", "bf16", "f32"]), lens_seed=rng.randrange(1 << 30))
        c["hi"] = c["mid"] * log_int(2, 16)
        c["prefixes"] = min(c["prefixes"], c["n"])
        budget = work(listed()[10])["flops"]
        while work(c)["flops"] > budget:
            if c["n"] > 1:
                c["n"] = max(1, c["n"] * 2 // 3)
                c["prefixes"] = min(c["prefixes"], c["n"])
            else:
                c["shared"], c["hi"] = max(16, c["shared"] // 2), max(16, c["hi"] // 2)
                c["mid"] = min(c["mid"], c["hi"])
    del c["name"]
    return c


def _batch(case):
    """Own lengths (host), and the requests' groups: prefix_start [p + 1], prefix lengths [p]."""
    rng = np.random.default_rng(case["lens_seed"])
    n, p = case["n"], case["prefixes"]
    own_len = np.clip(np.rint(np.exp(np.log(case["mid"]) + 0.8 * rng.standard_normal(n))), 1, case["hi"]).astype(np.int64)
    if p == 0:
        return own_len, np.zeros(1, np.int64), np.zeros(0, np.int64)
    # one prefix: everybody's; more: ragged groups and lengths, and one request in eight at the end without a prefix
    members = n if p == 1 else n - n // 8
    cuts = np.sort(rng.integers(0, members + 1, p - 1))
    start = np.concatenate([[0], cuts, [members]]).astype(np.int64)
    lens = np.full(p, case["shared"], np.int64)
    if p > 1:
        lens = np.maximum(1, (case["shared"] * (0.5 + rng.random(p)))).astype(np.int64)
    return own_len, start, lens


def _sizes(case):
    """Per request: group (or -1), shared tokens (whole blocks of the prefix), tokens in all."""
    own_len, start, lens = _batch(case)
    n = case["n"]
    group = np.full(n, -1, np.int64)
    for p in range(len(lens)):
        group[start[p]:start[p + 1]] = p
    whole = np.append(lens // BLOCK * BLOCK, 0)
    shared = whole[group]
    return group, shared, shared + own_len


def work(case):
    if case["kind"] == "rows":
        e, r = (4 if case["dtype"] == "f32" else 2), case["rows"]
        read = r * (case["hq"] + 2 * case["hkv"]) * case["d"] * e
        written = r * case["d"] * (case["hq"] * e + 2 * case["hkv"] * ELEM[case["dtype"]])
        return {"bytes": read + written + r * (8 + 4 * case["axes"]), "flops": r * (case["hq"] + case["hkv"]) * case["d"] * 8}
    group, shared, total = _sizes(case)
    n = case["n"]
    if case["kind"] == "tables":
        rows = int((total - shared).sum()) if case["new"] == 0 else int(np.minimum(case["new"], total - shared).sum())
        stride = int((total.max() + BLOCK - 1) // BLOCK)
        return {"bytes": n * (16 + 4 * stride + 8) + rows * 12, "flops": 0}
    _, start, lens = _batch(case)
    e, hq, hkv, d = ELEM[case["dtype"]], case["hq"], case["hkv"], case["d"]
    tokens = int((total - shared).sum()) + int((lens // BLOCK * BLOCK).sum())
    out = 4 if case["out"] == "f32" else 2
    return {"bytes": tokens * hkv * d * e * 2 + n * hq * d * (2 + out), "flops": int(total.sum()) * hq * d * 4}


# ---- the pools' format: views of a pool whose indices are (head, block, token of the block, channel) ------------------

def _k_index(t, c, dtype):
    """Element of a K block that holds channel c of token t."""
    if dtype == "fp8":
        return (((c // 64) * 4 + (c // 8) % 4) * 16 + t) * 16 + ((c // 32) % 2) * 8 + c % 8
    x = 16 // ELEM[dtype]
    return ((c // x) * 16 + t) * x + c % x


def _v_index(t, c, dtype):
    if dtype == "fp8":
        return ((c // 64) * 64 + (t // 4) * 16 + c % 16) * 16 + ((c // 16) % 4) * 4 + t % 4
    return (((c // 32) * 4 + t // 4) * 16 + c % 16) * 8 + ((c // 16) % 2) * 4 + t % 4


def _to_pool(rows, index, dtype):
    """Rows [tokens][heads][D] in the pool's format, one layer, flat."""
    tokens, heads, d = rows.shape
    t = torch.arange(BLOCK, device=rows.device)[:, None]
    c = torch.arange(d, device=rows.device)[None, :]
    at = index(t, c, dtype).reshape(-1)
    flat = rows.reshape(tokens // BLOCK, BLOCK, heads, d).permute(2, 0, 1, 3).reshape(heads, tokens // BLOCK, BLOCK * d)
    pool = torch.empty_like(flat)
    pool[:, :, at] = flat
    return pool.reshape(-1)


def _handle(state, case, *, k_pool, v_pool, tokens, n, hq, hkv, d, dtype, out):
    """The pool handle that a serving program keeps."""
    from paper_2512_09427_amd import binding as B
    args = dict(n_layers=1, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, kv_dtype={"f32": B.F32, "bf16": B.BF16, "fp8": B.FP8}[dtype],
                out_dtype={"f32": B.F32, "bf16": B.BF16}[out], main_tokens=tokens, safety_tokens=BLOCK, large_cap=BLOCK,
                boundaries=(BLOCK,), quantiles=((1, 2),), max_requests=max(n, 1))
    if dtype == "fp8":
        args.update(k_scale=FP8_SCALE, v_scale=FP8_SCALE)
    size = B.odma_workspace_bytes(B.make_config(**args)[0])
    ws = torch.empty(size, dtype=torch.uint8, device=DEV)
    state["B"] = B
    state["pool"] = B.Pool(*B.make_config(**args, k_pool=k_pool, v_pool=v_pool, workspace=ws))


def _dev(a, dtype):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV).to(dtype)


def _slabs(sizes, rng, gap=True):
    """Contiguous places for the given numbers of tokens, in a shuffled order: offsets, and the tokens they take in all."""
    caps = (np.asarray(sizes, np.int64) + BLOCK - 1) // BLOCK * BLOCK + (BLOCK if gap else 0)
    order = rng.permutation(len(caps))
    off = np.zeros(len(caps), np.int64)
    off[order] = np.cumsum(caps[order]) - caps[order]
    return off, max(int(caps.sum()), BLOCK)


def _prepare_tables(case, seed):
    rng = np.random.default_rng(seed)
    group, shared, total = _sizes(case)
    _, start, lens = _batch(case)
    n, p = case["n"], case["prefixes"]
    off, tokens = _slabs(np.concatenate([total - shared, lens]), rng)
    new = (total - shared) if case["new"] == 0 else np.minimum(case["new"], total - shared)
    rows = int(new.sum())
    s = dict(kind="tables", n=n, p=p, lengths=_dev(total, torch.int32), n_new=None if case["new"] == 1 else _dev(new, torch.int32),
             offsets=_dev(off[:n], torch.int64), prefix_start=_dev(start, torch.int32), prefix_offsets=_dev(off[n:], torch.int64),
             prefix_lengths=_dev(lens, torch.int32), stride=int((total.max() + BLOCK - 1) // BLOCK), max_rows=rows)
    s["block_table"] = torch.empty(n, s["stride"], dtype=torch.int32, device=DEV)
    s["row_start"] = torch.empty(n + 1, dtype=torch.int64, device=DEV)
    s["row_position"] = torch.empty(rows, dtype=torch.int32, device=DEV)
    s["row_slot"] = torch.empty(rows, dtype=torch.int64, device=DEV)
    if own:
        k = torch.empty((tokens + BLOCK) * 32, dtype=torch.bfloat16, device=DEV)
        _handle(s, case, k_pool=k, v_pool=torch.empty_like(k), tokens=tokens, n=n, hq=1, hkv=1, d=32, dtype="bf16", out="bf16")
    return s


def _prepare_rows(case, seed):
    rng = np.random.default_rng(seed)
    gen = torch.Generator(device=DEV).manual_seed(seed)
    rows, hq, hkv, d, dtype = case["rows"], case["hq"], case["hkv"], case["d"], case["dtype"]
    typ = INPUT[dtype]
    # what the projection leaves: queries, keys and values of a row side by side
    qkv = torch.randn(rows, (hq + 2 * hkv) * d, generator=gen, device=DEV)
    qkv = (qkv * (0.5 + 2.0 * torch.rand(rows, 1, generator=gen, device=DEV))).to(typ)
    # runs of rows are consecutive tokens (prompts); a run of 0: single tokens of a decode step
    run = case["run"] or 1
    runs = (rows + run - 1) // run
    counts = np.full(runs, run, np.int64)
    counts[-1] = rows - run * (runs - 1)
    shape = np.random.default_rng(rows)              # the pool's size is the case's, not the seed's
    first = shape.integers(0, 2 * BLOCK, runs) if case["run"] == 0 else shape.integers(0, 2, runs) * BLOCK
    base, tokens = _slabs(counts + first, rng, gap=False)
    j = np.arange(rows) - np.repeat(np.cumsum(counts) - counts, counts)
    slot = np.repeat(base + first, counts) + j
    pos = np.repeat(rng.integers(0, case["far"], runs), counts) + j
    if case["axes"] == 1:
        positions = pos[None]
    else:                                            # frames of 24 x 32 patches after the text
        positions = np.stack([pos // 768, pos // 32 % 24, pos % 32])
    rot = case["rot"]
    inv_freq = (1e6 ** (-np.arange(0, rot, 2) / rot)).astype(np.float32)
    pairs = rot // 2
    axis = np.zeros(pairs, np.int64) if case["axes"] == 1 else np.minimum(np.arange(pairs) * 8 // (3 * pairs), 2)
    s = dict(kind="rows", case=case, qkv=qkv, q=qkv[:, :hq * d], k=qkv[:, hq * d:(hq + hkv) * d], v=qkv[:, (hq + hkv) * d:],
             row_slot=_dev(slot, torch.int64), positions=_dev(positions, torch.int32), axis=_dev(axis, torch.int64),
             inv_freq=_dev(inv_freq, torch.float32), eps=1e-6)
    s["q_weight"], s["k_weight"] = ((1 + 0.2 * torch.randn(2, d, generator=gen, device=DEV)).to(typ).unbind(0) if case["norm"]
                                    else (None, None))
    s["q_out"] = torch.empty(rows, hq, d, dtype=typ, device=DEV)
    s["k_pool"] = torch.zeros(hkv * (tokens + BLOCK) * d, dtype=torch.uint8 if dtype == "fp8" else typ, device=DEV)
    s["v_pool"] = torch.zeros_like(s["k_pool"])
    if own:
        _handle(s, case, k_pool=s["k_pool"], v_pool=s["v_pool"], tokens=tokens, n=1, hq=hq, hkv=hkv, d=d, dtype=dtype,
                out="f32" if dtype == "f32" else "bf16")
        s["prep"] = s["B"].make_qk_prep(q_weight=s["q_weight"], k_weight=s["k_weight"], eps=s["eps"], rot_dim=rot,
                                        adjacent=case["adjacent"], inv_freq=s["inv_freq"], n_axes=case["axes"], axis=axis)
    return s


def _prepare_shared(case, seed):
    rng = np.random.default_rng(seed)
    gen = torch.Generator(device=DEV).manual_seed(seed)
    group, shared, total = _sizes(case)
    _, start, lens = _batch(case)
    n, p, hq, hkv, d, dtype = case["n"], case["prefixes"], case["hq"], case["hkv"], case["d"], case["dtype"]
    off, tokens = _slabs(np.concatenate([total - shared, lens]), rng)
    tokens += BLOCK
    own_off, pre_off = off[:n], off[n:]
    stride = int((total.max() + BLOCK - 1) // BLOCK)
    table = None
    if case["paged"]:                                # every block somewhere else
        place = rng.permutation(tokens // BLOCK)
        j = np.arange(stride)[None]
        in_prefix = j < (shared // BLOCK)[:, None]
        first = np.append(pre_off, 0)[group][:, None] // BLOCK
        table = np.where(in_prefix, first + j, own_off[:, None] // BLOCK + j - (shared // BLOCK)[:, None])
        table = place[np.where(j < ((total + BLOCK - 1) // BLOCK)[:, None], table, 0)]
    k, v = (torch.randn(tokens, hkv, d, generator=gen, device=DEV) for _ in range(2))
    k, v = ((x / FP8_SCALE).clamp(-448, 448).to(STORE[dtype]) if dtype == "fp8" else x.to(STORE[dtype]) for x in (k, v))
    raw = torch.uint8 if dtype == "fp8" else STORE[dtype]
    k, v = k.view(raw), v.view(raw)
    s = dict(kind="shared", case=case, n=n, p=p, rows_k=k, rows_v=v, q=torch.randn(n, hq, d, generator=gen, device=DEV).to(torch.bfloat16),
             group=_dev(group, torch.int64), shared=_dev(shared, torch.int64), lengths=_dev(total, torch.int32),
             offsets=_dev(own_off, torch.int64), prefix_start=_dev(start, torch.int32), prefix_offsets=_dev(pre_off, torch.int64),
             prefix_lengths=_dev(lens, torch.int32), stride=stride, table=None if table is None else _dev(table, torch.int32),
             most_members=max(int(np.diff(start).max()), 1), most_shared=max(int(shared.max()), BLOCK),
             most_own=int((total - shared).max()))
    s["out"] = torch.empty(n, hq, d, dtype={"f32": torch.float32, "bf16": torch.bfloat16}[case["out"]], device=DEV)
    s["k_pool"], s["v_pool"] = _to_pool(k, _k_index, dtype), _to_pool(v, _v_index, dtype)
    if own:
        _handle(s, case, k_pool=s["k_pool"], v_pool=s["v_pool"], tokens=tokens - BLOCK, n=n, hq=hq, hkv=hkv, d=d, dtype=dtype,
                out=case["out"])
    return s


def prepare(case, seed):
    return {"tables": _prepare_tables, "rows": _prepare_rows, "shared": _prepare_shared}[case["kind"]](case, seed)


# ---- plain forms --------------------------------------------------------------------------------------------------------

def _plain_tables(s):
    n, p, lengths, off = s["n"], s["p"], s["lengths"].long(), s["offsets"]
    ids = torch.arange(n, device=DEV)
    if p:
        group = torch.searchsorted(s["prefix_start"].long(), ids, right=True) - 1
        inside = (group >= 0) & (group < p)
        group = group.clamp(0, p - 1)
        shared = torch.where(inside, s["prefix_lengths"].long()[group] // BLOCK * BLOCK, 0)
        first = torch.where(inside, s["prefix_offsets"][group], 0)
    else:
        shared, first = torch.zeros_like(lengths), torch.zeros_like(off)
    j = torch.arange(s["stride"], device=DEV)[None]
    entry = torch.where(j < (shared // BLOCK)[:, None], (first // BLOCK)[:, None] + j,
                        ((off - shared) // BLOCK)[:, None] + j)
    table = torch.where(j < ((lengths + BLOCK - 1) // BLOCK)[:, None], entry, 0).int()
    new = lengths.clamp(max=1) if s["n_new"] is None else s["n_new"].long()
    row_start = torch.cat([torch.zeros(1, dtype=torch.int64, device=DEV), new.cumsum(0)])
    row = torch.arange(s["max_rows"], device=DEV)
    r = (torch.searchsorted(row_start, row, right=True) - 1).clamp(0, n - 1)
    position = lengths[r] - new[r] + row - row_start[r]
    slot = torch.where(position < shared[r], SLOT_SHARED, off[r] + position - shared[r])
    there = row < row_start[n]
    return table, row_start, torch.where(there, position, 0).int(), torch.where(there, slot, SLOT_NONE)


def _plain_norm(x, weight, eps):
    return x if weight is None else x * torch.rsqrt(x.square().mean(-1, keepdim=True) + eps) * weight.float()


def _plain_rotate(x, cos, sin, rot, adjacent):
    head, rest = x[..., :rot], x[..., rot:]
    a, b = (head[..., 0::2], head[..., 1::2]) if adjacent else (head[..., :rot // 2], head[..., rot // 2:])
    y = (a * cos - b * sin, b * cos + a * sin)
    y = torch.stack(y, -1).flatten(-2) if adjacent else torch.cat(y, -1)
    return torch.cat([y, rest], -1)


def _plain_write(pool, rows, slot, index, dtype, scale):
    d, heads = rows.shape[2], rows.shape[1]
    if dtype == "fp8":
        rows = (rows / scale).clamp(-448, 448)
    at = (slot // BLOCK)[:, None] * (BLOCK * d) + index((slot % BLOCK)[:, None], torch.arange(d, device=DEV)[None], dtype)
    pool = pool.view(heads, -1)
    stored = rows.to(STORE[dtype])
    if dtype == "fp8":
        stored = stored.view(torch.uint8)
    pool[:, at] = stored.permute(1, 0, 2)
    return pool.reshape(-1)


def _stored(pool, dtype):
    return pool.view(torch.float8_e4m3fn) if dtype == "fp8" else pool


def _plain_rows(s):
    c = s["case"]
    hq, hkv, d, dtype, rot = c["hq"], c["hkv"], c["d"], c["dtype"], c["rot"]
    x = s["qkv"].float().view(-1, hq + 2 * hkv, d)
    angle = s["positions"][s["axis"]].T.double() * s["inv_freq"].double()        # 64 bits: far positions
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    q = _plain_rotate(_plain_norm(x[:, :hq], s["q_weight"], s["eps"]), cos, sin, rot, c["adjacent"])
    k = _plain_rotate(_plain_norm(x[:, hq:hq + hkv], s["k_weight"], s["eps"]), cos, sin, rot, c["adjacent"])
    s["q_out"].copy_(q)
    kp = _plain_write(s["k_pool"], k, s["row_slot"], _k_index, dtype, FP8_SCALE)
    vp = _plain_write(s["v_pool"], x[:, hq + hkv:], s["row_slot"], _v_index, dtype, FP8_SCALE)
    return s["q_out"], _stored(kp, dtype), _stored(vp, dtype)


def _values(rows, slot, dtype):
    """The K or V rows [..][heads][D] of token slots, as stored values."""
    got = rows[slot]
    return got.view(torch.float8_e4m3fn) if dtype == "fp8" else got


def _plain_shared(s):
    """Two softmaxes with one reference: over the prefixes, group by group, and over every request's own tokens."""
    c, n, p = s["case"], s["n"], s["p"]
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    g, scale = hq // hkv, 1.0 / math.sqrt(d)
    unit = FP8_SCALE if c["dtype"] == "fp8" else 1.0
    q = s["q"].float()
    # prefixes: [group][head][member x g][token]
    i = torch.arange(s["most_members"], device=DEV)[None]
    member = s["prefix_start"].long()[:p, None] + i
    real = member < s["prefix_start"].long()[1:, None]
    member = member.clamp(max=n - 1)
    t = torch.arange(s["most_shared"], device=DEV)[None]
    held = t < (s["prefix_lengths"].long() // BLOCK * BLOCK)[:, None]
    if s["table"] is None:
        slot = s["prefix_offsets"][:, None] + t
    else:
        j = (t // BLOCK).clamp(max=s["stride"] - 1)
        slot = s["table"].long()[s["prefix_start"].long()[:p].clamp(max=n - 1)[:, None], j] * BLOCK + t % BLOCK
    slot = torch.where(held, slot, 0)
    kp = (_values(s["rows_k"], slot, c["dtype"]).float() * unit).permute(0, 2, 3, 1)
    vp = (_values(s["rows_v"], slot, c["dtype"]).float() * unit).permute(0, 2, 1, 3)
    qp = q[member].view(p, -1, hkv, g, d).permute(0, 2, 1, 3, 4).reshape(p, hkv, -1, d)
    sp = (qp @ kp.contiguous() * scale).masked_fill(~held[:, None, None], -math.inf)
    # own tokens: [request][head][g][token]
    t = torch.arange(s["most_own"], device=DEV)[None]
    own_len = s["lengths"].long() - s["shared"]
    held = t < own_len[:, None]
    if s["table"] is None:
        slot = s["offsets"][:, None] + t
    else:
        at = s["shared"][:, None] + t
        slot = s["table"].long().gather(1, (at // BLOCK).clamp(max=s["stride"] - 1)) * BLOCK + at % BLOCK
    slot = torch.where(held, slot, 0)
    ko = (_values(s["rows_k"], slot, c["dtype"]).float() * unit).permute(0, 2, 3, 1)
    vo = (_values(s["rows_v"], slot, c["dtype"]).float() * unit).permute(0, 2, 1, 3)
    so = (q.view(n, hkv, g, d) @ ko.contiguous() * scale).masked_fill(~held[:, None, None], -math.inf)
    # the prefix parts back in the requests' order
    mp = sp.amax(-1, keepdim=True)
    mp = torch.where(mp == -math.inf, 0.0, mp)
    wp = torch.exp(sp - mp)
    lp, op = wp.sum(-1, keepdim=True), wp @ vp.contiguous()

    def back(x, empty):
        x = x.view(p, hkv, -1, g, x.shape[-1]).permute(0, 2, 1, 3, 4)
        y = torch.full((n + 1, hkv, g, x.shape[-1]), empty, device=DEV)
        y[torch.where(real, member, n)] = x
        return y[:n]

    mp, lp, op = back(mp, -math.inf), back(lp, 0.0), back(op, 0.0)
    m = torch.maximum(so.amax(-1, keepdim=True), torch.where(lp > 0, mp, -math.inf))
    wo = torch.exp(so - m)
    f = torch.where(lp > 0, torch.exp(mp - m), 0.0)
    out = (wo @ vo.contiguous() + f * op) / (wo.sum(-1, keepdim=True) + f * lp)
    s["out"].copy_(out.view(n, hq, d))
    return s["out"]


# ---- one pass -------------------------------------------------------------------------------------------------------------

def _run_tables(s):
    if not own:
        return _plain_tables(s)
    s["pool"].odma_build_tables(s["n"], s["lengths"], s["n_new"], s["offsets"], s["p"], s["prefix_start"] if s["p"] else None,
                                s["prefix_offsets"] if s["p"] else None, s["prefix_lengths"] if s["p"] else None,
                                s["block_table"], s["stride"], s["max_rows"], s["row_start"], s["row_position"], s["row_slot"])
    return s["block_table"], s["row_start"], s["row_position"], s["row_slot"]


def _run_rows(s):
    if not own:
        return _plain_rows(s)
    c, stride = s["case"], s["qkv"].shape[1]
    s["pool"].odma_append_qkv(0, c["rows"], s["prep"], s["q"], stride, s["k"], stride, s["v"], stride, s["row_slot"],
                              s["positions"], s["q_out"])
    return s["q_out"], _stored(s["k_pool"], c["dtype"]), _stored(s["v_pool"], c["dtype"])


def _run_shared(s):
    if not own:
        return _plain_shared(s)
    s["pool"].odma_decode_attention_shared(0, s["n"], s["q"], s["p"], s["prefix_start"], s["prefix_offsets"], s["prefix_lengths"],
                                           s["offsets"], s["lengths"], s["table"], s["stride"] if s["table"] is not None else 0,
                                           s["out"])
    return s["out"]


def run(state):
    return {"tables": _run_tables, "rows": _run_rows, "shared": _run_shared}[state["kind"]](state)


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------------

def _exact_rows(case, s):
    hq, hkv, d, dtype, rot = case["hq"], case["hkv"], case["d"], case["dtype"], case["rot"]
    angle = torch.stack([s["positions"][a].double() for a in s["axis"].tolist()], 1) * s["inv_freq"].double()
    turn = torch.polar(torch.ones_like(angle), angle)[:, None]                   # e^(i angle): a rotation is a product

    def prepared(x, weight):
        x = x.double().reshape(x.shape[0], -1, d)
        if weight is not None:
            x = x / (x.pow(2).sum(-1, keepdim=True) / d + s["eps"]).sqrt() * weight.double()
        x = x.clone()
        at = torch.arange(rot // 2, device=DEV)
        i, j = (2 * at, 2 * at + 1) if case["adjacent"] else (at, at + rot // 2)
        z = torch.complex(x[..., i], x[..., j]) * turn
        x[..., i], x[..., j] = z.real, z.imag
        return x

    def pool_of(rows, index):
        elements = s["k_pool"].numel() // hkv
        pool = torch.zeros(hkv, elements, dtype=torch.float64, device=DEV)
        t, block = s["row_slot"] % BLOCK, s["row_slot"] // BLOCK
        for h in range(hkv):
            at = block[:, None] * BLOCK * d + index(t[:, None], torch.arange(d, device=DEV)[None], dtype)
            pool[h, at.reshape(-1)] = rows[:, h].reshape(-1) / (FP8_SCALE if dtype == "fp8" else 1.0)
        return pool.reshape(-1)

    v = s["v"].double().reshape(-1, hkv, d)
    return prepared(s["q"], s["q_weight"]), pool_of(prepared(s["k"], s["k_weight"]), _k_index), pool_of(v, _v_index)


def _exact_shared(case, s):
    n, hq, hkv, d = case["n"], case["hq"], case["hkv"], case["d"]
    group, shared, total = _sizes(case)
    unit = FP8_SCALE if case["dtype"] == "fp8" else 1.0
    if int(total.sum()) * hq * d > 2e11:
        return None
    first, own_first = s["prefix_offsets"].tolist(), s["offsets"].tolist()
    out = torch.empty(n, hq, d, dtype=torch.float64, device=DEV)
    for r in range(n):
        t = torch.arange(int(total[r]), device=DEV)
        if s["table"] is not None:
            slot = s["table"][r].long()[t // BLOCK] * BLOCK + t % BLOCK
        else:
            slot = own_first[r] + t - int(shared[r])
            if shared[r]:
                slot = torch.where(t < int(shared[r]), first[group[r]] + t, slot)
        k = (_values(s["rows_k"], slot, case["dtype"]).double() * unit).transpose(0, 1).repeat_interleave(hq // hkv, 0)
        v = (_values(s["rows_v"], slot, case["dtype"]).double() * unit).transpose(0, 1).repeat_interleave(hq // hkv, 0)
        score = (k * s["q"][r].double()[:, None]).sum(-1) / math.sqrt(d)
        out[r] = (torch.softmax(score, -1)[..., None] * v).sum(1)
    return out


def exact(case, seed):
    if case["kind"] == "tables":
        return None
    s = prepare(case, seed)
    return _exact_rows(case, s) if case["kind"] == "rows" else _exact_shared(case, s)
