"""Rotary positions with the append (flex_attn_rope_append) against the fp64
oracle: every geometry, both pairings, one to four axes, partial rotation,
padding, slots and positions out of range, strides, in place, captured."""
import numpy as np
import pytest
import torch

import oracle.rope_kv8 as RK
from paper_2606_04415_amd import flexattn as F

from gpu_common import log
from kv8_common import bf16, table

pytestmark = pytest.mark.gpu

# hq, hkv, dqk, dv, page
QWEN, D64, LATENT, SPLIT = (28, 4, 128, 128, 16), (15, 5, 64, 64, 64), (64, 1, 576, 512, 64), (16, 16, 192, 128, 64)


class Case:
    def __init__(self, geo, n, rot_begin=0, rot_dim=None, neighbours=False, sections=None, dealt=False, seed=1, gap=0,
                 pages=40):
        self.hq, self.hkv, self.dqk, self.dv, self.P = geo
        self.n, self.begin, self.rot = n, rot_begin, rot_dim or self.dqk
        self.neighbours, self.sections, self.dealt = neighbours, sections, dealt
        alias = self.dqk == 576
        r = np.random.RandomState(seed)
        self.axes = len(sections) if sections else 1
        self.max_pos = 5000
        self.tab = table(self.max_pos, self.rot)
        self.pos = r.randint(0, self.max_pos, size=(self.axes, n)).astype(np.int32)
        self.slots = r.permutation(pages * self.P)[:n].astype(np.int32)
        wide = [self.hq * self.dqk, self.hkv * self.dqk, 0 if alias else self.hkv * self.dv]
        row = bf16((n, sum(wide) + gap), seed)            # q, k and v of a token in one row
        self.q = row[:, :wide[0]].unflatten(1, (self.hq, self.dqk))
        self.k = row[:, wide[0]:wide[0] + wide[1]].unflatten(1, (self.hkv, self.dqk))
        self.v = None if alias else row[:, wide[0] + wide[1]:sum(wide)].unflatten(1, (self.hkv, self.dv))
        self.row, self.wide = row, wide
        self.kc = bf16((pages, self.P, self.hkv, self.dqk), seed + 1)
        self.vc = None if alias else bf16((pages, self.P, self.hkv, self.dv), seed + 2)
        self.shape = F.make_shape(self.hq, self.hkv, self.dqk, self.dv, self.P, 0.1, alias)

    def gpu(self):
        row = self.row.cuda()
        w = self.wide
        return dict(q=row[:, :w[0]].unflatten(1, (self.hq, self.dqk)),
                    k=row[:, w[0]:w[0] + w[1]].unflatten(1, (self.hkv, self.dqk)),
                    v=None if self.v is None else row[:, w[0] + w[1]:sum(w)].unflatten(1, (self.hkv, self.dv)),
                    kc=self.kc.cuda(), vc=None if self.vc is None else self.vc.cuda(), slots=torch.from_numpy(self.slots).cuda(),
                    pos=torch.from_numpy(self.pos).cuda(), tab=self.tab.cuda(), bad=torch.zeros(1, dtype=torch.int32, device="cuda"),
                    q_out=torch.full((self.n, self.hq, self.dqk), 7.0, dtype=torch.bfloat16, device="cuda"))

    def rope(self, g):
        return F.make_rope(g["tab"], g["pos"], rot_begin=self.begin, neighbours=self.neighbours, sections=self.sections,
                           dealt=self.dealt)

    def run(self, g=None, stream=None):
        g = g or self.gpu()
        rope = self.rope(g)
        args = F.make_rope_append_args(g["q"], g["q_out"], g["k"], g["v"], g["slots"], g["kc"], g["vc"], g["bad"])
        F.flex_attn_rope_append(self.shape, rope, args, stream=stream)
        g["keep"] = (rope, args)
        return g

    def check(self, g, what):
        tab = self.tab.double().numpy()
        ok = (self.pos >= 0).all(0) & (self.pos < self.max_pos).all(0)
        slot_ok = (self.slots >= 0) & (self.slots < self.kc.shape[0] * self.P)
        live = ok & slot_ok
        pos = np.where(ok[None], self.pos, 0)

        def turn(x):
            y = x.double().numpy()
            return RK.rotate(y, tab, pos, self.begin, self.neighbours, self.sections, self.dealt)

        def near(got, x, name):
            """fp32: each product and the sum round, 3 * 2^-24 of |x c| + |y s| <= |x| + |y|; then bf16, 2^-8."""
            ref = turn(x)
            mag = np.abs(x.double().numpy()).max(-1, keepdims=True)
            bound = 2.0 ** -8 * np.abs(ref) + 6 * 2.0 ** -24 * mag
            err = np.abs(got.double().cpu().numpy() - ref)
            assert (err <= bound)[live].all(), f"{what}: {name} off by {(err - bound)[live].max():.3g} more than its bound"

        near(g["q_out"], self.q, "q")
        assert (g["q_out"].cpu().view(torch.int16)[torch.from_numpy(~live)] ==
                torch.tensor(7.0, dtype=torch.bfloat16).view(torch.int16)).all(), f"{what}: a skipped token's query was written"
        kc = g["kc"].cpu().view(-1, self.hkv, self.dqk)
        got = torch.zeros_like(self.k)
        got[torch.from_numpy(live)] = kc[torch.from_numpy(self.slots[live]).long()]
        near(got, self.k, "k")
        b, e = self.begin, self.begin + self.rot               # the columns that pass are copied bit for bit
        for c in (slice(0, b), slice(e, None)):
            assert torch.equal(got[live][..., c].view(torch.int16), self.k[live][..., c].contiguous().view(torch.int16))
            assert torch.equal(g["q_out"].cpu()[live][..., c].contiguous().view(torch.int16),
                               self.q[live][..., c].contiguous().view(torch.int16))
        rest = np.setdiff1d(np.arange(kc.shape[0]), self.slots[live])
        assert torch.equal(kc[rest].view(torch.int16), self.kc.view(kc.shape)[rest].view(torch.int16)), f"{what}: other rows changed"
        if self.vc is not None:
            vc = self.vc.clone().view(-1, self.hkv, self.dv)
            vc[torch.from_numpy(self.slots[live]).long()] = self.v[live].contiguous()
            assert torch.equal(g["vc"].cpu().view(torch.int16).flatten(), vc.view(torch.int16).flatten()), f"{what}: values"
        bad = int(((self.slots >= 0) & ~live).sum())
        assert int(g["bad"].item()) == bad, f"{what}: bad_count {int(g['bad'].item())}, not {bad}"
        log(f"  {what}: {self.n} tokens, {int(live.sum())} written, {bad} out of range")


@pytest.mark.parametrize("geo,kw", [
    (QWEN, {}), (QWEN, dict(neighbours=True)), (QWEN, dict(rot_dim=64)), (QWEN, dict(rot_dim=32, rot_begin=40)),
    (D64, {}), (D64, dict(rot_dim=16, rot_begin=8, neighbours=True)),
    (LATENT, dict(rot_begin=512, rot_dim=64, neighbours=True)), (LATENT, dict(rot_begin=512, rot_dim=64)),
    (SPLIT, dict(rot_begin=128, rot_dim=64, neighbours=True)),
    ((4, 1, 64, 64, 16), {}), ((40, 8, 128, 128, 64), {}), ((1, 1, 128, 128, 16), {}),
])
@pytest.mark.parametrize("n", [1, 3, 37])
def test_rotation(geo, kw, n):
    log(f"rope append {geo} {kw}, {n} tokens")
    c = Case(geo, n, seed=10 + n, **kw)
    g = c.run()
    torch.cuda.synchronize()
    c.check(g, "rope")


@pytest.mark.parametrize("geo,sections,dealt,kw", [
    (QWEN, [16, 24, 24], False, {}), (QWEN, [24, 20, 20], True, {}), (QWEN, [64, 0], False, {}),
    (QWEN, [1, 2, 61], False, dict(neighbours=True)), (QWEN, [16, 16, 16, 16], True, {}), (D64, [3, 13, 9, 7], False, {}),
    (D64, [12, 10, 10], True, dict(neighbours=True)), (LATENT, [12, 10, 10], False, dict(rot_begin=512, rot_dim=64)),
])
def test_several_axes(geo, sections, dealt, kw):
    log(f"rope append {geo}, axes {sections} dealt {dealt} {kw}")
    c = Case(geo, 29, sections=sections, dealt=dealt, seed=5, **kw)
    g = c.run()
    torch.cuda.synchronize()
    c.check(g, "axes")


def test_equal_axes_are_one_axis():
    """Positions alike on all axes give the one-axis result bit for bit."""
    one = Case(QWEN, 50, seed=3)
    three = Case(QWEN, 50, sections=[16, 24, 24], seed=3)
    three.pos = np.repeat(one.pos, 3, 0)
    three.slots = one.slots
    a, b = one.run(), three.run()
    torch.cuda.synchronize()
    assert torch.equal(a["q_out"].view(torch.int16), b["q_out"].view(torch.int16))
    assert torch.equal(a["kc"].view(torch.int16), b["kc"].view(torch.int16))


@pytest.mark.parametrize("geo,kw", [(QWEN, {}), (LATENT, dict(rot_begin=512, rot_dim=64, neighbours=True)),
                                    (D64, dict(sections=[10, 11, 11]))])
def test_padding_and_bad_tokens_are_skipped(geo, kw):
    c = Case(geo, 33, seed=8, gap=24, **kw)
    c.slots[[0, 7, 32]] = [-1, -5, -2 ** 31]                       # padding
    c.slots[[3, 9]] = [c.kc.shape[0] * c.P, 2 ** 31 - 1]           # outside the pool
    c.pos[-1, [3, 4, 20]] = [-1, c.max_pos, -2 ** 31]              # one at fault on both counts
    c.pos[0, 7] = c.max_pos                                        # padding may hold anything
    g = c.run()
    torch.cuda.synchronize()
    c.check(g, "skips")


def test_in_place_equals_out_of_place():
    c = Case(QWEN, 21, seed=4)
    g = c.run()
    h = c.gpu()
    h["q"] = h["q"].contiguous()
    h["q_out"] = h["q"]
    c.run(h)
    torch.cuda.synchronize()
    assert torch.equal(g["q_out"].view(torch.int16), h["q"].view(torch.int16))
    assert torch.equal(g["kc"].view(torch.int16), h["kc"].view(torch.int16))


def test_empty_call_and_far_positions():
    c = Case(QWEN, 4, seed=2)
    c.n = 0
    for f in ("q", "k", "v", "row"):
        setattr(c, f, getattr(c, f)[:0])
    c.slots, c.pos = c.slots[:0], c.pos[:, :0]
    g = c.run()
    torch.cuda.synchronize()
    assert torch.equal(g["kc"].cpu().view(torch.int16), c.kc.view(torch.int16))
    far = Case(QWEN, 9, seed=6, rot_dim=32)
    far.max_pos = 1 << 20
    far.tab = table(far.max_pos, 32)
    far.pos[0, :3] = [far.max_pos - 1, 0, far.max_pos - 77]
    g = far.run()
    torch.cuda.synchronize()
    far.check(g, "far")


def test_on_another_stream_and_captured():
    c = Case(QWEN, 64, seed=12)
    ref = c.run()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    g = c.gpu()
    torch.cuda.synchronize()
    c.run(g, stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(g["q_out"].view(torch.int16), ref["q_out"].view(torch.int16))
    h = c.gpu()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run(h)
    for k in range(3):
        h["q_out"].fill_(float(k))
        h["kc"].copy_(c.kc)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(h["q_out"].view(torch.int16), ref["q_out"].view(torch.int16)), f"replay {k}"
        assert torch.equal(h["kc"].view(torch.int16), ref["kc"].view(torch.int16)), f"replay {k}"
