"""odma_append_qkv against norms and rotations in 64 bits: every type, head size, pairing and number of axes, rows in runs that
begin anywhere in a block, single rows, rows that are not there.  The whole pool is read back: slots of other tokens keep what
they held."""
import math

import numpy as np
import pytest
import torch

import workloads as wl
from paper_2512_09427_amd import binding as B

DEV = "cuda"
pytestmark = pytest.mark.gpu
KV = {"f32": B.F32, "bf16": B.BF16, "fp8": B.FP8}
K_SCALE, V_SCALE = 2.0 ** -5, 2.0 ** -6
# half a step of the type, relative (E4M3: and half of its smallest step, absolute)
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "fp8": 2.0 ** -4}


class Case:
    def __init__(self, kvd, hq, hkv, d, tokens, slots, *, rot, adjacent=False, axes=1, norm=True, layers=1, seed=0, far=100000, packed=True,
                 edit=None):
        gen = torch.Generator().manual_seed(seed)
        self.kvd, self.hq, self.hkv, self.d, self.tokens, self.rot, self.adjacent = kvd, hq, hkv, d, tokens, rot, adjacent
        self.typ = torch.float32 if kvd == "f32" else torch.bfloat16
        n = self.n = len(slots)
        self.slots = torch.tensor(slots, dtype=torch.int64)
        if packed:
            x = torch.randn(n, (hq + 2 * hkv) * d, generator=gen) * (0.1 + 3 * torch.rand(n, 1, generator=gen))
            if edit:
                edit(x)
            x = x.to(self.typ).to(DEV)
            self.q, self.k, self.v = x[:, :hq * d], x[:, hq * d:(hq + hkv) * d], x[:, (hq + hkv) * d:]
        else:
            self.q, self.k, self.v = (torch.randn(n, h * d, generator=gen).to(self.typ).to(DEV) for h in (hq, hkv, hkv))
        self.weights = [(1 + 0.3 * torch.randn(d, generator=gen)).to(self.typ).to(DEV) if norm else None for _ in range(2)]
        self.inv_freq = (10000.0 ** (-torch.arange(0, rot, 2).double() / max(rot, 1))).float().to(DEV)
        self.positions = torch.randint(0, far, (axes, n), generator=gen, dtype=torch.int32).to(DEV)
        self.axis = [(3 * f + f // 5) % axes for f in range(rot // 2)]
        self.prep = B.make_qk_prep(q_weight=self.weights[0], k_weight=self.weights[1], eps=1e-5, rot_dim=rot, adjacent=adjacent,
                                   inv_freq=self.inv_freq if rot else None, n_axes=axes, axis=self.axis)
        elems = layers * hkv * (tokens + 16) * d
        raw = torch.uint8 if kvd == "fp8" else self.typ
        self.k_pool, self.v_pool = (torch.full((elems,), v, dtype=raw, device=DEV) for v in ((7, 9) if kvd == "fp8" else (-3.0, 5.0)))
        args = dict(n_layers=layers, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, kv_dtype=KV[kvd], out_dtype=B.F32, main_tokens=tokens,
                    safety_tokens=16, large_cap=16, boundaries=(16,), quantiles=((1, 2),), max_requests=1)
        if kvd == "fp8":
            args.update(k_scale=K_SCALE, v_scale=V_SCALE)
        self.pool = B.Pool(*B.make_config(**args, k_pool=self.k_pool, v_pool=self.v_pool))
        self.q_out = torch.full((n, hq, d), -7.0, dtype=self.typ, device=DEV)

    def call(self, layer=0, stream=None, q_out=None):
        self.pool.odma_append_qkv(layer, self.n, self.prep, self.q, self.q.stride(0), self.k, self.k.stride(0), self.v, self.v.stride(0),
                                  self.slots.to(DEV), self.positions if self.rot else None, self.q_out if q_out is None else q_out, stream)

    def stored(self, layer=0):
        """All rows of a layer of the pools, as stored."""
        k = torch.empty(self.tokens + 16, self.hkv, self.d, dtype=self.k_pool.dtype, device=DEV)
        v = torch.empty_like(k)
        self.pool.odma_gather_kv(layer, 0, self.tokens + 16, None, k, v)
        torch.cuda.synchronize()
        return k.cpu(), v.cpu()

    def reference(self, x, heads, weight):
        """64 bits, and the length of every channel's pair (or its own size), which bounds what rounding the turn can do."""
        x = x.cpu().double().view(self.n, heads, self.d)
        if weight is not None:
            x = x * (x.square().mean(-1, keepdim=True) + float(np.float32(1e-5))).rsqrt() * weight.cpu().double()
        x, size = x.clone(), x.abs()
        for f in range(self.rot // 2):
            i, j = (2 * f, 2 * f + 1) if self.adjacent else (f, f + self.rot // 2)
            angle = (self.positions.cpu()[self.axis[f]].double() * float(self.inv_freq[f]))[:, None]
            a, b = x[..., i].clone(), x[..., j].clone()
            x[..., i], x[..., j] = a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin()
            size[..., i] = size[..., j] = torch.sqrt(a * a + b * b)
        return x, size

    def check(self, before, layer=0, q_out=None):
        there, kept = self.slots != -1, (self.slots >= 0) & (self.slots < self.tokens + 16)
        there &= self.slots < self.tokens + 16
        # fp32 arithmetic: a norm's sum, root and products and a turn, each a few 2^-24; the fraction of a turn 2^-26
        # around zero, and the 64-bit product of a position (three roundings)
        slack = 16 * 2.0 ** -24 + 3 * 2.0 ** -53 * float(self.positions.abs().max())
        ref, size = self.reference(self.q, self.hq, self.weights[0])
        got = (self.q_out if q_out is None else q_out).cpu().double().view(self.n, self.hq, self.d)
        half = HALF["f32" if self.kvd == "f32" else "bf16"]
        assert ((got - ref).abs() <= half * ref.abs() + slack * size)[there].all(), (got - ref).abs()[there].max()
        if q_out is None:
            assert (got[~there] == -7).all()                       # rows that are not there
        k, v = self.stored(layer)
        slots = self.slots[kept]
        ref, size = self.reference(self.k, self.hkv, self.weights[1])
        got, vgot, vref = k[slots], v[slots], self.v.cpu().view(self.n, self.hkv, self.d)[kept]
        if self.kvd == "fp8":
            ref, size = (ref / K_SCALE).clamp(-448, 448), size / K_SCALE
            got = torch.from_numpy(wl.e4m3_bits_to_f32(got.numpy())).double()
            vref = torch.from_numpy(wl.f32_to_e4m3_bits((vref.float() / V_SCALE).numpy()))
        tiny = 2.0 ** -10 if self.kvd == "fp8" else 0.0
        bound = HALF[self.kvd] * ref.abs() + slack * size + tiny
        assert ((got.double() - ref[kept]).abs() <= bound[kept]).all(), (got.double() - ref[kept]).abs().max()
        assert torch.equal(vgot, vref)                               # values are moved (E4M3: rounded once)
        rest = torch.ones(self.tokens + 16, dtype=torch.bool)
        rest[slots] = False
        for now, was in zip((k, v), before):
            assert torch.equal(now[rest], was[rest])

    def run(self):
        before = self.stored()
        self.call()
        self.check(before)


def mixed_slots(seed=0, tokens=512):
    """Runs that begin anywhere in a block, cross blocks and end anywhere, single tokens, rows that are not there or shared, in
    rows that no tile boundary respects."""
    rng = np.random.default_rng(seed)
    free, out = list(range(0, tokens, 64)), []
    rng.shuffle(free)
    for base, (first, count) in zip(free, [(0, 40), (3, 21), (14, 5), (16, 16), (1, 1), (62, 2), (4, 33), (0, 3)]):
        out += [base + first + i for i in range(count)]
        out += [[], [-1], [-2, -2], [-1, -2, -1]][rng.integers(0, 4)]
    return out


SHAPES = [("bf16", 28, 4, 128), ("bf16", 4, 2, 64), ("bf16", 3, 1, 32), ("bf16", 5, 5, 96), ("bf16", 8, 1, 256), ("bf16", 2, 1, 160),
          ("f32", 2, 1, 64), ("f32", 7, 1, 128), ("f32", 3, 3, 224), ("f32", 9, 3, 32), ("fp8", 28, 4, 128), ("fp8", 1, 1, 128)]


@pytest.mark.parametrize("kind", ["halves, normed", "adjacent", "partial, three axes", "norm alone", "neither"])
@pytest.mark.parametrize("kvd,hq,hkv,d", SHAPES)
def test_rows_anywhere(kvd, hq, hkv, d, kind):
    kw = {"halves, normed": dict(rot=d), "adjacent": dict(rot=d, adjacent=True, norm=False),
          "partial, three axes": dict(rot=d // 2 // 8 * 8 if d > 32 else 24, axes=3, far=3000), "norm alone": dict(rot=0),
          "neither": dict(rot=0, norm=False)}[kind]
    Case(kvd, hq, hkv, d, 512, mixed_slots(d), seed=d, **kw).run()


@pytest.mark.parametrize("kvd,hq,hkv,d", [("bf16", 28, 4, 128), ("fp8", 28, 4, 128), ("f32", 2, 1, 64)])
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 64, 257])
def test_decode_steps(kvd, hq, hkv, d, n):
    """One row per request, each in a block of its own, at every place of a block."""
    Case(kvd, hq, hkv, d, 32 * n, [32 * i + (7 * i) % 32 for i in range(n)], rot=d, seed=n).run()


@pytest.mark.parametrize("kvd,hq,hkv,d,adjacent,axes", [("bf16", 28, 4, 128, False, 1), ("bf16", 12, 2, 64, True, 4), ("fp8", 4, 4, 128, False, 3),
                                                        ("f32", 2, 2, 256, False, 1)])
def test_long_prompts(kvd, hq, hkv, d, adjacent, axes):
    """Thousands of rows: work-groups with all heads of a tile."""
    slots = list(range(5, 5 + 9001)) + list(range(9200, 9200 + 8000))
    Case(kvd, hq, hkv, d, 18000 // 16 * 16, slots, rot=d, adjacent=adjacent, axes=axes).run()


@pytest.mark.parametrize("far", [2 ** 20, 2 ** 24, 2 ** 31 - 1])
def test_far_positions(far):
    """The angle itself: in fp32 a position of a million times a frequency of 1 is whole, its fraction of a turn off by 2^-6."""
    c = Case("f32", 4, 1, 64, 64, list(range(33)), rot=64, norm=False, far=far)
    c.positions[0, :2] = torch.tensor([far - 1, far], dtype=torch.int64).to(torch.int32).to(DEV)
    c.run()


def test_negative_positions_and_four_axes():
    c = Case("bf16", 4, 2, 128, 64, list(range(20)), rot=128, axes=4)
    c.positions -= 50000
    c.run()


def test_separate_rows_in_another_layer_and_in_place():
    c = Case("bf16", 6, 2, 128, 64, list(range(3, 40)), rot=128, layers=3, packed=False)
    before = [c.stored(i) for i in range(3)]
    c.call(layer=1)
    c.check(before[1], layer=1)
    for i in (0, 2):
        assert all(torch.equal(a, b) for a, b in zip(c.stored(i), before[i]))
    kept, c.q = c.q.clone(), c.q.clone()
    c.call(layer=1, q_out=c.q)                                      # queries in place
    got, c.q = c.q, kept
    assert torch.equal(got.view(-1), c.q_out.view(-1))


def test_a_query_of_zeros_and_of_huge_values():
    """A head of zeros stays one (eps), values near the end of the range do not overflow where their norm does not."""
    def edit(x):
        x[0] = 0
        x[1, :128] = 1e15
        x[2, 128:] = 1e-20

    c = Case("bf16", 2, 1, 128, 32, list(range(8)), rot=128, edit=edit)
    c.run()
    assert (c.q_out[0] == 0).all()


def test_fp8_keeps_to_its_range():
    """Beyond +-448 the largest value, infinities too; NaN stays NaN."""
    def edit(x):
        x[0, 128:] = 100.0
        x[1, 128:] = -math.inf
        x[2, 128:] = math.nan

    c = Case("fp8", 1, 1, 128, 32, list(range(4)), rot=0, norm=False, edit=edit)
    c.call()
    k, v = c.stored()
    for x in (k, v):
        assert (x[0] == 0x7e).all() and (x[1] == 0xfe).all() and ((x[2] & 0x7f) == 0x7f).all()


def test_a_row_with_nan_touches_no_other():
    def edit(x):
        x[5] = math.nan

    c = Case("bf16", 4, 2, 128, 64, list(range(16)), rot=128, edit=edit)
    clean = Case("bf16", 4, 2, 128, 64, list(range(16)), rot=128)
    c.call()
    clean.call()
    keep = [i for i in range(16) if i != 5]
    assert torch.equal(c.q_out[keep], clean.q_out[keep]) and torch.isnan(c.q_out[5]).all()
    for x, y in zip(c.stored(), clean.stored()):
        assert torch.equal(x[keep], y[keep])


def test_slots_past_the_pool_are_not_there():
    c = Case("bf16", 4, 2, 64, 64, [0, 80, 1 << 40, -(1 << 40), 79, 5], rot=64)
    before = c.stored()
    c.call()
    q_out = c.q_out.cpu()
    assert (q_out[[1, 2]] == -7).all() and (q_out[[0, 4, 5]] != -7).any(-1).all()
    k, v = c.stored()
    rest = [i for i in range(80) if i not in (0, 79, 5)]
    assert torch.equal(k[rest], before[0][rest]) and torch.equal(v[rest], before[1][rest])


def test_captured_and_on_a_stream_of_its_own():
    c = Case("bf16", 28, 4, 128, 256, mixed_slots(1, 256)[:60], rot=128)
    slots = c.slots = c.slots.to(DEV)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        c.call()
    side.synchronize()
    want, stored = c.q_out.clone(), c.stored()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.call()
    for _ in range(3):
        c.q_out.fill_(-7)
        c.k_pool.fill_(-3.0)
        c.v_pool.fill_(5.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(c.q_out, want) and all(torch.equal(a, b) for a, b in zip(c.stored(), stored))
    assert c.slots is slots
