"""The append into an 8-bit cache (flex_attn_kv8_append) against its oracle:
codes and scale bytes bit for bit (the rotation on fp32 products, as defined),
queries under the bound of their rounding."""
import numpy as np
import pytest
import torch

import oracle.rope_kv8 as RK
from paper_2606_04415_amd import flexattn as F

from gpu_common import log
from kv8_common import batch, bf16, cache8, table, to_gpu

pytestmark = pytest.mark.gpu

QWEN, D64, ONE, WIDE = (28, 4, 128, 16), (15, 5, 64, 64), (4, 1, 64, 16), (40, 20, 128, 64)


class Case:
    def __init__(self, geo, ns, ls, seed=1, rope=True, pad=0, sizes=0.7, max_pos=4096, positions=False, width=0, **kw):
        self.hq, self.hkv, self.d, self.P = geo
        self.kw, self.rope_on = kw, rope
        self.bt, self.ls, self.qsl, pages = batch(ns, ls, self.P, seed, width=width)
        self.n = int(self.qsl[-1]) + pad
        r = np.random.RandomState(seed)
        size = torch.from_numpy(np.exp(sizes * r.randn(self.n, 1, 1)).astype(np.float32))
        self.q = bf16((self.n, self.hq, self.d), seed)
        self.k = (bf16((self.n, self.hkv, self.d), seed + 1).float() * size).to(torch.bfloat16)
        self.v = (bf16((self.n, self.hkv, self.d), seed + 2).float() * size).to(torch.bfloat16)
        self.codes = cache8(pages, self.P, self.hkv, self.d, seed)
        self.max_pos = max_pos
        self.rot = kw.pop("rot_dim", self.d)
        self.tab = table(max_pos, self.rot)
        own = np.concatenate([np.arange(L - n, L) for n, L in zip(ns, ls)] + [np.zeros(pad, dtype=int)]).astype(np.int32)
        sections = kw.get("sections")
        self.pos = np.stack([own] if not sections else [r.randint(0, max_pos, self.n) for _ in sections]).astype(np.int32)
        self.given = positions or bool(sections)
        self.shape = F.make_shape(self.hq, self.hkv, self.d, self.d, self.P, 0.1)

    def gpu(self):
        k, v, s = to_gpu(*[x.copy() for x in self.codes])
        return dict(q=self.q.cuda(), k=self.k.cuda(), v=self.v.cuda(), kc=k, vc=v, sc=s, bt=torch.from_numpy(self.bt).cuda(),
                    ls=torch.from_numpy(self.ls).cuda(), qsl=torch.from_numpy(self.qsl).cuda(), tab=self.tab.cuda(),
                    pos=torch.from_numpy(self.pos).cuda(), bad=torch.zeros(1, dtype=torch.int32, device="cuda"),
                    q_out=torch.full((self.n, self.hq, self.d), 7.0, dtype=torch.bfloat16, device="cuda"))

    def run(self, g=None, stream=None):
        g = g or self.gpu()
        rope = F.make_rope(g["tab"], g["pos"] if self.given else None, **self.kw) if self.rope_on else None
        q = (g["q"], g["q_out"]) if self.rope_on else (None, None)
        args = F.make_kv8_append_args(g["k"], g["v"], g["bt"], g["ls"], g["qsl"], g["kc"], g["vc"], g["sc"], *q, bad_count=g["bad"])
        F.flex_attn_kv8_append(self.shape, rope, args, stream=stream)
        g["keep"] = (rope, args)
        return g

    def reference(self):
        """(k codes, v codes, scales) after the append."""
        k, v = self.k.float().numpy(), self.v.float().numpy()
        if self.rope_on:
            k = RK.rotate(k, self.tab.numpy(), self.pos, self.kw.get("rot_begin", 0), self.kw.get("neighbours", False),
                          self.kw.get("sections"), self.kw.get("dealt", False), dtype=np.float32)
        kc, vc, sc = self.codes
        with np.errstate(invalid="ignore", over="ignore"):
            rk, ks = RK.kv8_append(kc, sc[..., 0], k, self.bt, self.ls, self.qsl, self.P)
            rv, vs = RK.kv8_append(vc, sc[..., 1], v, self.bt, self.ls, self.qsl, self.P)
        return rk, rv, np.stack([ks, vs], -1)

    def check(self, g, what):
        torch.cuda.synchronize()
        ref = self.reference()
        for name, got, want in zip(("scales", "k", "v"), (g["sc"], g["kc"], g["vc"]), (ref[2], ref[0], ref[1])):
            got = got.view(torch.uint8).cpu().numpy()
            if name != "scales":   # NaN is one value, whatever its sign
                got, want = (np.where((x & 127) == 127, 127, x) for x in (got, want))
            assert np.array_equal(got, want), f"{what}: {name} differs in {(got != want).sum()} of {got.size} bytes"
        if self.rope_on:
            T = int(self.qsl[-1])
            x = self.q[:T].double().numpy()
            turned = RK.rotate(x, self.tab.double().numpy(), self.pos[:, :T], self.kw.get("rot_begin", 0),
                               self.kw.get("neighbours", False), self.kw.get("sections"), self.kw.get("dealt", False))
            # 3 * 2^-24 of |x c| + |y s| in fp32, then bf16
            bound = 2.0 ** -8 * np.abs(turned) + 6 * 2.0 ** -24 * np.abs(x).max(-1, keepdims=True)
            got = g["q_out"].double().cpu().numpy()
            assert (np.abs(got[:T] - turned) <= bound).all(), f"{what}: q"
            assert (got[T:] == 7.0).all(), f"{what}: a padding row was written"
        log(f"  {what}: {self.n} tokens, codes, scales and queries agree")


RAGGED = ([1, 1, 1, 1, 5, 16, 0, 33, 1, 70, 1], [1, 16, 17, 100, 5, 48, 9, 40, 129, 70, 64])


@pytest.mark.parametrize("geo", [QWEN, D64, ONE, WIDE])
@pytest.mark.parametrize("kw", [{}, dict(rope=False), dict(neighbours=True), dict(rot_dim=32, rot_begin=16)])
def test_ragged_batch(geo, kw):
    log(f"kv8 append {geo} {kw}")
    c = Case(geo, *RAGGED, seed=3, pad=3, **kw)
    c.check(c.run(), "ragged")


@pytest.mark.parametrize("sections,dealt", [([16, 24, 24], False), ([24, 20, 20], True), ([5, 59], False)])
def test_several_axes(sections, dealt):
    c = Case(QWEN, *RAGGED, seed=5, sections=sections, dealt=dealt)
    c.check(c.run(), f"axes {sections}")


@pytest.mark.parametrize("geo,ns,axes", [
    (QWEN, [2100], 1), (QWEN, [4099], 1), (D64, [1500, 1500, 1500], 3), (ONE, [1] * 500 + [1600], 1), (ONE, [1] * 500 + [3700], 3),
    (ONE, [1] * 130 + [8200], 1)])
def test_many_tokens(geo, ns, axes):
    """Tokens by two waves and by one: prompts, and single tokens among them."""
    log(f"kv8 append of {sum(ns)} tokens {geo} on {axes} axes")
    kw = dict(sections=[8, 12, 12]) if axes > 1 else {}
    c = Case(geo, ns, [n + 7 * i % 40 for i, n in enumerate(ns)], seed=len(ns), pad=5, max_pos=9000, **kw)
    c.check(c.run(), "many tokens")


def test_given_positions_are_the_tokens_own():
    a, b = Case(QWEN, *RAGGED, seed=6), Case(QWEN, *RAGGED, seed=6, positions=True)
    ga, gb = a.run(), b.run()
    a.check(ga, "own")
    b.check(gb, "given")


@pytest.mark.parametrize("B", [1, 63, 64, 65, 300, 5000])
def test_sequence_search(B):
    """Batches on both sides of the search's 64 probes, with empty sequences among them."""
    r = np.random.RandomState(B)
    ns = r.choice([0, 1, 1, 1, 2], size=B)
    ns[-1] = 1
    ls = ns + r.randint(0, 20, size=B)
    c = Case(ONE, ns.tolist(), ls.tolist(), seed=B, rope=B < 1000)
    log(f"kv8 append of {B} sequences, {c.n} tokens")
    c.check(c.run(), "search")


def test_scale_grows_and_stays():
    """A block that fills up token by token: scales only grow, earlier rows
    keep their values up to the rounding at the new scale, and each step is the
    oracle's."""
    c = Case(QWEN, [1], [1], seed=9, sizes=0.0)
    g = c.gpu()
    sizes = [2.0 ** -20, 1.0, 0.5, 30.0, 1e-3, 1e4, 1.0, 1e30, 0.0, 2.0 ** 100]
    for i, f in enumerate(sizes):
        c.ls = np.array([i + 1], dtype=np.int32)
        c.pos = np.array([[i]], dtype=np.int32)
        c.k, c.v = bf16((1, 4, 128), 20 + i, f), bf16((1, 4, 128), 40 + i, f)
        g.update(k=c.k.cuda(), v=c.v.cuda(), ls=torch.from_numpy(c.ls).cuda())
        c.run(g)
        c.check(g, f"row {i}, size {f:g}")
        c.codes = tuple(x.view(torch.uint8).cpu().numpy() for x in (g["kc"], g["vc"], g["sc"]))
    assert (c.codes[2][c.bt[0, 0], 0] >= 127 + 80).all()


def test_zero_rows_infinities_and_nans():
    c = Case(ONE, [20, 1, 3], [20, 18, 3], seed=2, rope=False)
    c.k[:16] = 0                                  # a block of zeros: the least scale
    c.k[20, 0, 5], c.v[20, 0, 6] = float("inf"), float("-inf")
    c.k[21, 0, 1], c.v[22, 0, 0] = float("nan"), float("nan")
    c.v[21:24] = float("inf")                     # nothing finite in a block of its own
    g = c.run()
    c.check(g, "special values")
    sc = g["sc"].view(torch.uint8).cpu().numpy()
    assert sc[c.bt[0, 0], 0, 0, 0] == 10


def test_exact_powers_and_the_largest_code():
    """Magnitudes on both sides of 448 * 2^k, where the scale changes."""
    c = Case(ONE, [16] * 5, [16] * 5, seed=2, rope=False)
    c.k[:], c.v[:] = 0, 0
    for i, x in enumerate([448.0, 450.0, 446.0, 2.0 ** -126, 3.3e38]):
        c.k[16 * i + 3, 0, 7], c.v[16 * i, 0, 0] = x, -x
    g = c.run()
    c.check(g, "edges")
    sc = g["sc"].view(torch.uint8).cpu().numpy()
    assert [int(sc[c.bt[i, 0], 0, 0, 0]) for i in range(4)] == [127, 128, 127, 10]


@pytest.mark.parametrize("geo", [QWEN, D64])
def test_every_scale_byte_that_a_block_can_have(geo):
    """A block that holds a row takes one more, at each of the 256 scale bytes:
    those that an empty cache has or that the append writes, and the rest. New
    rows from tiny to the type's largest."""
    for size in (2.0 ** -100, 1.0, 2.0 ** 126):
        c = Case(geo, [1] * 256, [2 + i % 15 for i in range(256)], seed=6, rope=False)
        c.k = (c.k.float().clamp(-2, 2) / 2 * size).to(torch.bfloat16)
        c.v = (c.v.float().clamp(-2, 2) / 2 * size).to(torch.bfloat16)
        for s in range(256):
            c.codes[2][c.bt[s, 0], 0] = s
        c.check(c.run(), f"rows of {size:g}")


def test_bad_pages_and_positions_are_skipped_and_counted():
    c = Case(QWEN, [1, 40, 1, 1], [30, 40, 5, 50], seed=4, positions=True)
    good = c.reference()
    c.bt[0, 1] = c.codes[0].shape[0]              # sequence 0's token: outside the pool
    c.bt[1, 1] = -3                               # tokens 16 .. 31 of sequence 1
    c.pos[0, 41] = c.max_pos                      # sequence 2's token
    g = c.run()
    torch.cuda.synchronize()
    assert int(g["bad"].item()) == 18
    got = g["kc"].view(torch.uint8).cpu().numpy()
    want = c.codes[0].copy()
    for s, t0, t1 in ((1, 0, 16), (1, 32, 40), (3, 0, 50)):   # pages of the tokens that are in range
        for p in range(t0 // 16, -(-t1 // 16)):
            want[c.bt[s, p]] = good[0][c.bt[s, p]]
    live = np.ones(want.shape[0], dtype=bool)
    live[c.bt[2, 0]] = False                      # its one row is unspecified
    assert np.array_equal(got[live], want[live])
    q = g["q_out"].cpu()
    skipped = [0] + list(range(17, 33)) + [41]
    assert (q[skipped] == 7.0).all() and (q[[1, 16, 33, 42]] != 7.0).any(-1).any(-1).all()


@pytest.mark.parametrize("geo", [QWEN, ONE])
@pytest.mark.parametrize("ns,ls", [([1, 1], [17, 1]), ([3, 16, 1], [19, 16, 20]), ([20, 2], [36, 40])])
def test_a_block_of_skipped_tokens_keeps_its_scale(geo, ns, ls):
    """Every token's position is outside the table: codes, scales and queries stay
    as they are, in blocks whose first row is among the tokens as in others."""
    c = Case(geo, ns, ls, seed=4, positions=True)
    c.pos[:] = np.where(np.arange(c.n) % 2, -1, c.max_pos)[None]
    g = c.run()
    torch.cuda.synchronize()
    assert int(g["bad"].item()) == c.n
    for n, was in zip(("kc", "vc", "sc"), c.codes):
        assert np.array_equal(g[n].view(torch.uint8).cpu().numpy(), was), n
    assert (g["q_out"].cpu() == 7.0).all()


def test_tokens_past_the_calls_are_left_out():
    """n_tokens below query_start_loc's end: the tokens past it are not appended."""
    c = Case(QWEN, [1, 30], [9, 30], seed=7, rope=False)
    g = c.gpu()
    args = F.make_kv8_append_args(g["k"][:20], g["v"][:20], g["bt"], g["ls"], g["qsl"], g["kc"], g["vc"], g["sc"])
    F.flex_attn_kv8_append(c.shape, None, args)
    torch.cuda.synchronize()
    got = g["kc"].view(torch.uint8).cpu().numpy()
    assert np.array_equal(got[c.bt[1, 1], 3:], c.codes[0][c.bt[1, 1], 3:])
    assert not np.array_equal(got[c.bt[1, 1], :3], c.codes[0][c.bt[1, 1], :3])


@pytest.mark.parametrize("geo,ns,ls,first", [
    (QWEN, [5, 1, 20, 1], [5, 40, 33, 17], 1), (QWEN, [3, 2, 1], [3, 16, 100], 2), (ONE, [9, 30], [9, 64], 1),
    (D64, [1] * 80 + [7], [20] * 80 + [50], 70), (ONE, [4200, 40, 3], [4200, 41, 19], 1)])
@pytest.mark.parametrize("rope", [True, False])
def test_tokens_before_the_first_sequence_are_padding(geo, ns, ls, first, rope):
    """A part of a batch, its query_start_loc starting above 0: the tokens of the
    sequences left out are no one's. Nothing of theirs is written, nothing counted."""
    log(f"kv8 append {geo}: sequences from {first} of {len(ns)}, rope {rope}")
    c = Case(geo, ns, ls, seed=13, rope=rope, pad=2, max_pos=8192)
    c.bt, c.ls, c.qsl = c.bt[first:].copy(), c.ls[first:].copy(), c.qsl[first:].copy()
    g = c.run()
    torch.cuda.synchronize()
    assert int(g["bad"].item()) == 0
    want = c.reference()
    for n, ref in zip(("kc", "vc", "sc"), want):
        got = g[n].view(torch.uint8).cpu().numpy()
        assert np.array_equal(got, ref), f"{n} differs in {(got != ref).sum()} of {ref.size} bytes"
    if rope:
        q, t0, t1 = g["q_out"].cpu(), int(c.qsl[0]), int(c.qsl[-1])
        assert (q[:t0] == 7.0).all() and (q[t1:] == 7.0).all() and (q[t0:t1] != 7.0).any(-1).any(-1).all()


def test_strided_caches_and_rows():
    """A cache that is part of a larger one (both of K and V, other layers'
    pages between) and rows of one projection: the gaps keep their bytes."""
    c = Case(D64, *RAGGED, seed=8, width=5)
    g = c.gpu()
    pages = c.codes[0].shape[0]
    both = torch.full((pages, 2, c.P, c.hkv + 1, c.d + 16), 0x55, dtype=torch.uint8, device="cuda")
    for i, n in enumerate(("kc", "vc")):
        both[:, i, :, :c.hkv, :c.d] = g[n].view(torch.uint8)
        g[n] = both[:, i, :, :c.hkv, :c.d].view(torch.float8_e4m3fn)
    scales = torch.full((pages, 3, c.P // 16, c.hkv, 2), 0x55, dtype=torch.uint8, device="cuda")
    scales[:, 1] = g["sc"].view(torch.uint8)
    g["sc"] = scales[:, 1].view(torch.float8_e8m0fnu)
    rows = torch.zeros((c.n, c.hq + 2 * c.hkv + 1, c.d), dtype=torch.bfloat16, device="cuda")
    for n, at, m in (("q", 0, c.hq), ("k", c.hq, c.hkv), ("v", c.hq + c.hkv, c.hkv)):
        rows[:, at:at + m] = g[n]
        g[n] = rows[:, at:at + m]
    c.run(g)
    c.check(g, "strided")
    assert (both[:, :, :, c.hkv:] == 0x55).all() and (both[..., c.d:] == 0x55).all()
    assert (scales[:, 0] == 0x55).all() and (scales[:, 2] == 0x55).all()


def test_far_pages():
    """Pages past 5 GiB of codes, with slots 80 KiB apart."""
    c = Case(D64, *RAGGED, seed=12)
    g = c.gpu()
    used, gap = c.codes[0].shape[0], 80 << 10
    far = (5 << 30) // (c.P * gap) + 1
    pool = torch.zeros((far + used) * c.P * gap, dtype=torch.uint8, device="cuda")
    wide = pool.as_strided((far + used, c.P, c.hkv, c.d), (c.P * gap, gap, c.d, 1))
    wide[far:] = g["kc"].view(torch.uint8)
    big = dict(g, kc=wide.view(torch.float8_e4m3fn), bt=g["bt"] + far)
    for n in ("vc", "sc"):
        x = torch.zeros((far + used, *g[n].shape[1:]), dtype=torch.uint8, device="cuda")
        x[far:] = g[n].view(torch.uint8)
        big[n] = x.view(g[n].dtype)
    c.run(big)
    torch.cuda.synchronize()
    assert all(not big[n][:far].view(torch.uint8).any() for n in ("kc", "vc", "sc"))
    c.check(dict(big, **{n: big[n][far:] for n in ("kc", "vc", "sc")}), "far")


def test_twice_is_once_and_captured():
    """The same append again changes nothing, and replays of a captured one,
    with other work between, give what the eager call gives."""
    c = Case(QWEN, *RAGGED, seed=11)
    ref = c.run()
    c.check(c.run(ref), "twice")
    h = c.gpu()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run(h)
    fresh = c.gpu()
    for k in range(3):
        for n in ("kc", "vc", "sc"):
            h[n].view(torch.uint8).copy_(fresh[n].view(torch.uint8))
        h["q_out"].fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        c.check(h, f"replay {k}")
    side = torch.cuda.Stream()
    g = c.gpu()
    torch.cuda.synchronize()
    c.run(g, stream=side.cuda_stream)
    side.synchronize()
    c.check(g, "another stream")
