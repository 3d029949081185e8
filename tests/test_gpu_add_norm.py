"""odma_add_norm against its formula in 64 bits: both types of rows and of the residual, every way to deal a row out to waves, with and
without norm of the block, gate and outputs, strides, rows that are not there, in place, streams and captured calls."""
import math

import pytest
import torch

from paper_2512_09427_amd import binding as B

DEV = "cuda"
pytestmark = pytest.mark.gpu
TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}        # half a step, relative
GATES = {"none": B.GATE_NONE, "value": B.GATE_VALUE, "sigmoid": B.GATE_SIGMOID}


def pool(typ, tokens=64):
    kv = torch.zeros(2 * (tokens + 16) * 32, dtype=TYPE[typ], device=DEV)
    t = B.F32 if typ == "f32" else B.BF16
    return B.Pool(*B.make_config(n_layers=1, n_q_heads=2, n_kv_heads=2, head_dim=32, kv_dtype=t, out_dtype=t, main_tokens=tokens, safety_tokens=16,
                                 large_cap=16, boundaries=(16,), quantiles=((1, 2),), max_requests=1, k_pool=kv, v_pool=kv.clone()))


class Case:
    def __init__(self, typ, res, rows, width, *, post=True, gate="none", one_gate=False, next_=True, block=True, rs=1.0, bs=1.0, eps=1e-6, pad=0,
                 seed=0, slots=None, edit=None):
        gen = torch.Generator().manual_seed(seed)
        self.typ, self.res, self.rows, self.width, self.rs, self.bs, self.slots = typ, res, rows, width, rs, bs, slots
        self.gate_kind, self.post, self.next_ = gate, post and block, next_

        def normal(*shape):
            return torch.randn(*shape, generator=gen)

        blk, old = normal(rows, width + pad), normal(rows, width + pad) * (0.2 + 4 * torch.rand(rows, 1, generator=gen))
        if edit:
            edit(blk, old)
        self.block, self.old = blk.to(TYPE[typ]).to(DEV) if block else None, old.to(TYPE[res]).to(DEV)
        self.wb = (1 + 0.3 * normal(width)).to(TYPE[typ]).to(DEV) if self.post else None
        self.wn = (1 + 0.3 * normal(width)).to(TYPE[typ]).to(DEV) if next_ else None
        self.gate = None if gate == "none" else (2 * normal(1 if one_gate else rows, width + pad)).to(TYPE[typ]).to(DEV)
        self.eps = float(torch.tensor(eps, dtype=torch.float32))
        self.how = B.make_add_norm(width=width, block_weight=self.wb, next_weight=self.wn, gate=self.gate, gate_kind=GATES[gate],
                                   gate_stride=0 if one_gate or gate == "none" else width + pad, eps=eps, residual_scale=rs, block_scale=bs,
                                   residual_dtype=B.F32 if res == "f32" else B.BF16)
        self.pool = pool(typ)
        self.out = torch.full((rows, width + pad), -7.0, dtype=TYPE[res], device=DEV)
        self.x = torch.full((rows, width), -7.0, dtype=TYPE[typ], device=DEV) if next_ else None
        self.stride = width + pad

    def run(self, stream=None, keep=True):
        self.pool.odma_add_norm(self.rows, self.how, self.block, self.stride if self.block is not None else 0, self.old, self.stride, self.slots,
                                self.out if keep else None, self.x, stream)
        return self

    def reference(self):
        w, d = self.width, torch.float64
        old = self.old[:, :w].cpu().to(d)
        b, loose = torch.zeros_like(old), torch.zeros_like(old)
        # fp32: a sum of squares is off by its terms one after the other in a lane (32 at most), those of the joining and a
        # product each, half of which reaches the root; root and products a step or two each
        norm = 40 * 2.0 ** -24
        if self.block is not None:
            b = self.block[:, :w].cpu().to(d)
            rel = torch.zeros_like(b)
            if self.post:
                b = b * (b.square().mean(-1, keepdim=True) + self.eps).rsqrt() * self.wb.cpu().to(d)
                rel = rel + norm
            if self.gate_kind != "none":
                g = self.gate[:, :w].cpu().to(d)
                b = b * (torch.sigmoid(g) if self.gate_kind == "sigmoid" else g)
                rel = rel + (8 + 4 * g.abs()) * 2.0 ** -24          # exponent, exponential, reciprocal, product
            loose = b.abs() * (rel + 2.0 ** -23) * abs(self.bs)
        r = self.rs * old + self.bs * b
        loose = loose + 2.0 ** -23 * ((self.rs * old).abs() + (self.bs * b).abs())
        x, loose_x = None, None
        if self.next_:
            inv = (r.square().mean(-1, keepdim=True) + self.eps).rsqrt()
            wn = self.wn.cpu().to(d)
            x = r * inv * wn
            # (what the row's own error does to its root: at most its mean relative to the root mean square)
            drift = (loose.square().mean(-1, keepdim=True)).sqrt() * inv
            loose_x = x.abs() * (norm + drift) + loose * inv * wn.abs()
        return r, loose, x, loose_x

    def check(self, keep=True, there=None):
        torch.cuda.synchronize()
        r, lr, x, lx = self.reference()
        there = torch.ones(self.rows, dtype=torch.bool) if there is None else there
        got = self.out.cpu().double()
        if keep:
            err = (got[:, :self.width] - r).abs()
            assert (err <= HALF[self.res] * r.abs() + lr + 1e-38)[there].all(), err[there].max()
            assert (got[:, self.width:] == -7).all() and (got[~there] == -7).all()
        else:
            assert (got == -7).all()
        if self.next_:
            got = self.x.cpu().double()
            err = (got - x).abs()
            assert (err <= HALF[self.typ] * x.abs() + lx * 1.01 + 1e-38)[there].all(), err[there].max()
            assert (got[~there] == -7).all()


TYPES = [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")]


# few rows: a wave for every 512 channels, up to 16, then several pieces each; many rows: fewer waves, more pieces each
@pytest.mark.parametrize("typ,res", TYPES)
@pytest.mark.parametrize("rows,width", [(1, 8), (3, 64), (5, 504), (2, 512), (7, 520), (3, 1032), (4, 2048), (2, 3584), (3, 4096), (2, 4104), (1, 8192),
                                        (2, 8200), (2, 16384), (1, 20000), (1, 32768), (1025, 8), (1030, 520), (1027, 1400), (1024, 2048),
                                        (1029, 3584), (1025, 4104), (1025, 8200)])
def test_widths(rows, width, typ, res):
    Case(typ, res, rows, width, gate="value", seed=width).run().check()


@pytest.mark.parametrize("typ,res", TYPES)
@pytest.mark.parametrize("rows,width", [(16400, 520), (49170, 2056), (1030, 4104), (1030, 8192)])
def test_many_rows(rows, width, typ, res):
    """Fewer waves to a row, with more pieces each."""
    Case(typ, res, rows, width, gate="none" if rows > 20000 else "sigmoid", seed=width).run().check()


@pytest.mark.parametrize("typ,res", TYPES)
@pytest.mark.parametrize("rows", [5, 1031])
@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("gate,one", [("none", False), ("value", False), ("value", True), ("sigmoid", False), ("sigmoid", True)])
def test_forms(gate, one, post, rows, typ, res):
    for next_ in (True, False):
        Case(typ, res, rows, 1096, post=post, gate=gate, one_gate=one, next_=next_, rs=0.75, bs=-0.3, eps=1e-3, pad=16, seed=2).run().check()
    c = Case(typ, res, rows, 1096, post=post, gate=gate, one_gate=one, rs=2.0, bs=0.25)
    c.run(keep=False).check(keep=False)                         # the residual is not kept


@pytest.mark.parametrize("typ,res", TYPES)
def test_in_front_of_the_first_block(typ, res):
    Case(typ, res, 9, 776, block=False).run(keep=False).check(keep=False)
    Case(typ, res, 9, 776, block=False, rs=3.0, pad=8).run().check()


@pytest.mark.parametrize("typ,res", TYPES)
@pytest.mark.parametrize("rows,width", [(6, 3584), (1040, 2056)])
def test_in_place(rows, width, typ, res):
    c = Case(typ, res, rows, width, gate="sigmoid")
    c.run()
    torch.cuda.synchronize()
    out, x = c.out.clone(), c.x.clone()
    # the new residual over the old one, x over the block's output
    c.pool.odma_add_norm(rows, c.how, c.block, width, c.old, width, None, c.old, c.block)
    torch.cuda.synchronize()
    assert torch.equal(c.old, out) and torch.equal(c.block, x)


@pytest.mark.parametrize("rows", [12, 1030])
def test_rows_that_are_not_there(rows):
    kinds = torch.tensor([0, B.SLOT_NONE, 79, B.SLOT_SHARED, 80, 1 << 40])
    slots = kinds[torch.arange(rows) % 6]
    for width in (512, 1024, 4000):
        def edit(blk, old):
            blk[slots == B.SLOT_NONE] = math.nan
        c = Case("bf16", "f32", rows, width, slots=slots.to(DEV), edit=edit, gate="value").run()
        c.check(there=(slots != B.SLOT_NONE) & (slots < 80))


def test_small_and_large_rows():
    """Rows of zeros, of squares near both ends of fp32's range; an infinity and a NaN stay in their row."""
    def edit(blk, old):
        blk[0], old[0] = 0, 0
        blk[1], old[1] = blk[1] * 1e-17, old[1] * 1e-17
        blk[2], old[2] = blk[2] * 1e16, old[2] * 1e16
        blk[3], old[3] = blk[3] * 1e-16, old[3] * 1e-16
    for post in (False, True):
        Case("f32", "f32", 5, 1024, post=post, eps=0.0 if not post else 1e-30, edit=lambda b, o: (edit(b, o), b[0].fill_(1e-3), o[0].fill_(1e-3))).run().check()
        Case("bf16", "bf16", 5, 1024, post=post, eps=1e-6, edit=edit).run().check()

    def spoil(blk, old):
        blk[1, 5], old[3, 7] = math.inf, math.nan
    for rows in (5, 1025):
        clean, c = Case("bf16", "bf16", rows, 640), Case("bf16", "bf16", rows, 640, edit=spoil)
        clean.run(), c.run()
        torch.cuda.synchronize()
        rest = [r for r in range(rows) if r not in (1, 3)]
        assert torch.equal(c.x[rest], clean.x[rest]) and torch.equal(c.out[rest], clean.out[rest])
        assert torch.isnan(c.x[3]).all() and torch.isnan(c.x[1]).any()


def test_far_rows():
    rows, width, stride = 5, 64, 1 << 29
    c = Case("bf16", "bf16", rows, width, seed=3)
    flat = [torch.zeros(rows * stride, dtype=torch.bfloat16, device=DEV) for _ in range(3)]
    for f, t in zip(flat, (c.block, c.old, c.out)):
        f.view(rows, stride)[:, :width] = t
    c.pool.odma_add_norm(rows, c.how, flat[0], stride, flat[1], stride, None, flat[2], c.x)
    c.out = flat[2].view(rows, stride)[:, :width].clone()
    c.check()


@pytest.mark.parametrize("rows", [3, 2000])
def test_streams_and_captured_calls(rows):
    a, b = (Case("bf16", "f32", rows, 3584, gate="sigmoid", seed=s) for s in (1, 2))
    want = []
    for c in (a, b):
        c.run()
        torch.cuda.synchronize()
        want.append((c.out.clone(), c.x.clone()))
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    for c in (a, b):
        c.out.fill_(1), c.x.fill_(1)
    torch.cuda.synchronize()
    a.run(one), b.run(two)
    torch.cuda.synchronize()
    for c, w in zip((a, b), want):
        assert torch.equal(c.out, w[0]) and torch.equal(c.x, w[1])
    # captured: a residual that runs on in place, against eager calls
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.pool.odma_add_norm(rows, a.how, a.block, a.width, a.old, a.width, None, a.old, a.x)
    eager, x = a.old.clone(), torch.empty_like(a.x)
    for i in range(4):
        graph.replay()
        a.pool.odma_add_norm(rows, a.how, a.block, a.width, eager, a.width, None, eager, x)
        torch.cuda.synchronize()
        assert torch.equal(a.old, eager) and torch.equal(a.x, x)
        a.block.mul_(0.5)
