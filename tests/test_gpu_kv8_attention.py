"""Attention over an 8-bit cache against its definition in 64 bits, within
bounds derived from the roundings that are made (kv8_common.check_attention).
Slots and blocks that no sequence uses hold NaN codes and NaN scales."""
import numpy as np
import pytest
import torch

import oracle.rope_kv8 as RK
from paper_2606_04415_amd import flexattn as F

from gpu_common import log
from kv8_common import attend64, batch, bf16, cache8, check_attention, poison, scale_of, to_gpu

pytestmark = pytest.mark.gpu

CALLS = {"decode": F.flex_attn_decode_kv8, "prefill": F.flex_attn_prefill_kv8}


class Case:
    def __init__(self, hq, hkv, d, P, ns, ls, seed=1, spread=3, width=0, q_scale=2.0):
        self.hq, self.hkv, self.d, self.P = hq, hkv, d, P
        self.ns, self.bt_ls = ns, ls
        self.bt, self.ls, self.qsl, pages = batch(ns, ls, P, seed, width=width)
        self.k, self.v, self.s = cache8(pages, P, hkv, d, seed, spread)
        poison(self.k, self.v, self.s, self.bt, ls, P)
        self.q = bf16((int(self.qsl[-1]), hq, d), seed, q_scale)
        self.shape = F.make_shape(hq, hkv, d, d, P, scale_of(d))

    def gpu(self):
        k, v, s = to_gpu(self.k, self.v, self.s)
        return dict(q=self.q.cuda(), k=k, v=v, s=s, bt=torch.from_numpy(self.bt).cuda(), ls=torch.from_numpy(self.ls).cuda(),
                    qsl=torch.from_numpy(self.qsl).cuda())

    def plan(self, **opts):
        return F.PagedAttention(self.shape, F.make_opts(kv_bits=8, **opts), self.qsl, self.ls, self.bt.shape[1])

    def run(self, call="serial", g=None, pa=None, corun=None, with_lse=True, **opts):
        g, pa = g or self.gpu(), pa or self.plan(**opts)
        out, lse = pa.alloc_out(g["q"], with_lse)
        out.fill_(float("nan"))
        if lse is not None:
            lse.fill_(float("nan"))
        args = pa.kv8_args(g["q"], g["k"], g["v"], g["s"], g["bt"], g["ls"], g["qsl"], out, lse)
        if call in CALLS:
            CALLS[call](pa.plan, args)
        else:
            F.flex_attn_mixed_kv8(pa.plan, args, F.FLEX_MODE_CORUN if call == "corun" else F.FLEX_MODE_SERIAL, corun=corun)
        torch.cuda.synchronize()
        return out.cpu(), None if lse is None else lse.cpu()

    def values(self):
        return RK.values(self.k, self.s[..., 0]), RK.values(self.v, self.s[..., 1])

    def reference(self):
        if not hasattr(self, "ref"):
            self.ref = attend64(self.q, *self.values(), self.bt, self.ls, self.qsl, np.float64(np.float32(scale_of(self.d))))
        return self.ref

    def check(self, out, lse, what):
        check_attention(out, lse, self.reference(), self.ls, self.qsl, self.d, what)


DECODES = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100, 127, 128, 129, 300, 1000, 2049]


@pytest.mark.parametrize("hq,hkv,d,P", [(28, 4, 128, 16), (28, 4, 128, 64), (15, 5, 64, 16), (32, 8, 64, 64), (4, 1, 64, 16),
                                        (16, 1, 128, 16), (32, 2, 128, 64), (8, 8, 128, 64), (6, 3, 64, 64), (20, 20, 64, 16),
                                        (24, 12, 128, 16)])
@pytest.mark.parametrize("opts", [{}, dict(min_split_tokens=64)])
def test_decode(hq, hkv, d, P, opts):
    log(f"kv8 decode {hq}/{hkv} d{d} page {P} {opts}")
    c = Case(hq, hkv, d, P, [1] * len(DECODES), DECODES, seed=hq + d)
    c.check(*c.run("decode", **opts), "decode")


@pytest.mark.parametrize("hq,hkv,d,P", [(28, 4, 128, 16), (32, 8, 64, 64), (32, 8, 128, 16), (4, 1, 64, 16)])
@pytest.mark.parametrize("count,top", [(1, 1), (3, 128), (40, 256), (600, 20)])
def test_decode_of_short_sequences(hq, hkv, d, P, count, top):
    """Ranges of whole sequences: one each, or several of every length after each other."""
    log(f"kv8 decode {hq}/{hkv} d{d} page {P}: {count} of up to {top}")
    c = Case(hq, hkv, d, P, [1] * count, [top] + [1 + (37 * i) % top for i in range(count - 1)], seed=count)
    assert c.plan().plan.info["n_split_seqs"] == 0
    c.check(*c.run("decode"), "short")


@pytest.mark.parametrize("hq,hkv,d,P", [(10, 5, 128, 16), (18, 9, 64, 64), (48, 6, 128, 64), (17, 17, 64, 16), (32, 8, 128, 16)])
def test_decode_in_several_columns(hq, hkv, d, P):
    """Rows of more than 512 bytes: work-groups of uneven groups of heads, pieces
    and whole sequences, merged by columns and by rows."""
    log(f"kv8 decode columns {hq}/{hkv} d{d} page {P}")
    c = Case(hq, hkv, d, P, [1] * len(DECODES), DECODES, seed=hq + d)
    assert c.plan().plan.info["decode_wg_width"] == -(-hkv * d // 512)
    c.check(*c.run("decode"), "columns")
    c.check(*c.run("decode", min_split_tokens=2048), "whole sequences")
    c = Case(hq, hkv, d, P, [1, 1], [3000, 17], seed=hq)
    c.check(*c.run("decode"), "many pieces")


@pytest.mark.parametrize("hq,hkv,d,P", [(28, 4, 128, 16), (28, 4, 128, 64), (15, 5, 64, 16), (32, 8, 64, 64), (4, 1, 64, 16),
                                        (16, 1, 128, 64), (8, 8, 128, 16), (24, 12, 128, 64)])
def test_prefill(hq, hkv, d, P):
    ns = [2, 3, 5, 31, 32, 33, 64, 65, 130, 7, 0, 2]
    ls = [2, 40, 5, 31, 64, 97, 64, 200, 130, 700, 12, 33]
    log(f"kv8 prefill {hq}/{hkv} d{d} page {P}")
    c = Case(hq, hkv, d, P, ns, ls, seed=hq + d)
    c.check(*c.run("prefill"), "prefill")


@pytest.mark.parametrize("d,P", [(128, 16), (64, 64)])
def test_mixed_leaves_the_rest_alone(d, P):
    """Both phases, sequences with nothing new among them, no log-sum-exp; rows
    of the other phase stay as they were in the calls of one phase."""
    ns, ls = [1, 40, 0, 1, 3, 1, 0], [90, 100, 50, 1, 3, 513, 0]
    c = Case(14, 2, d, P, ns, ls, seed=4)
    out, _ = c.run("serial", with_lse=False)
    c.check(out, None, "mixed")
    dec, _ = c.run("decode")
    pre, _ = c.run("prefill")
    single = torch.from_numpy(np.repeat(np.array(ns) == 1, ns))
    assert dec[~single].isnan().all() and pre[single].isnan().all()
    both = torch.where(single[:, None, None], dec, pre)
    assert torch.equal(both.view(torch.int16), out.view(torch.int16))


@pytest.mark.parametrize("hq,hkv,d,P,ns,ls", [(28, 4, 128, 16, [1, 1, 300, 1, 20, 1], [3000, 17, 700, 2500, 90, 129]),
                                              (32, 8, 64, 64, [1, 150, 1, 1], [900, 150, 4000, 5])])
@pytest.mark.parametrize("tail", [0, -1])
def test_corun_equals_serial(hq, hkv, d, P, ns, ls, tail):
    c = Case(hq, hkv, d, P, ns, ls, seed=7)
    corun = F.Corun(160, 96)
    try:
        pa = c.plan(cus_decode=96, min_split_tokens=64, decode_tail=tail)
        g = c.gpu()
        stream = torch.cuda.Stream()
        a = c.run("serial", g, pa)
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            for k in range(3):
                b = c.run("corun", g, pa, corun)
                assert torch.equal(a[0].view(torch.int16), b[0].view(torch.int16)) and torch.equal(a[1], b[1]), f"step {k}"
    finally:
        corun.close()
    c.check(*a, "co-run plan")


@pytest.mark.parametrize("spread,q_scale", [(1, 0.0), (1, 0.01), (3, 20.0), (12, 2.0)])
def test_scores_from_flat_to_sharp(spread, q_scale):
    """All scores alike, and softmaxes that one key takes; scales that differ by up to 2^11 between blocks."""
    c = Case(28, 4, 128, 16, [1, 1, 50, 1], [700, 33, 90, 64], seed=5, spread=spread, q_scale=q_scale)
    c.check(*c.run(min_split_tokens=64), f"spread {spread} queries {q_scale}")


def test_single_key_is_its_value():
    c = Case(28, 4, 128, 16, [1, 1], [1, 1], seed=6)
    out, _ = c.run()
    v = c.values()[1]
    for s in range(2):
        want = torch.from_numpy(np.repeat(v[c.bt[s, 0], 0], 7, 0)).to(torch.bfloat16)
        assert torch.equal(out[s], want)


def test_all_codes_and_scales_reach_the_output():
    """One key a sequence, its value row every finite code, at every scale of
    the append's range: code * scale exactly."""
    d, hkv = 128, 2
    ks = list(range(10, 240, 7))
    c = Case(hkv, hkv, d, 16, [1] * len(ks), [1] * len(ks), seed=1)
    row = np.array([x for x in range(256) if (x & 127) != 127], dtype=np.uint8)
    for s, b in enumerate(ks):
        c.v[c.bt[s, 0], 0] = np.stack([row[:128], row[126:]])
        c.s[c.bt[s, 0], 0, :, 1] = b
    out, _ = c.run()
    v = c.values()[1]
    want = torch.from_numpy(np.stack([v[c.bt[s, 0], 0] for s in range(len(ks))])).float()
    assert torch.equal(out.float(), want)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,ks", [(1, list(range(0, 10)) + list(range(240, 255))), (2, list(range(0, 10)) + list(range(240, 246)))])
def test_scale_bytes_at_the_ends(d, n, ks):
    """Bytes that the append does not write, or only for the largest values: byte
    0 is 2^-127, tiny values are subnormal ones, values from 2^128 on infinite. n
    new tokens with like keys and values (one: decode, two: prefill, whose
    second sums two halves)."""
    hkv = 256 // d
    c = Case(hkv, hkv, d, 16, [n] * len(ks), [n] * len(ks), seed=1)
    row = np.array([x for x in range(256) if (x & 127) != 127], dtype=np.uint8)
    for s, b in enumerate(ks):
        c.k[c.bt[s, 0], :n] = 0
        c.v[c.bt[s, 0], :n] = np.concatenate([row, row[:2]]).reshape(hkv, d)
        c.s[c.bt[s, 0], 0, :, 1] = b
    out, _ = c.run()
    v = c.values()[1]
    want = torch.from_numpy(np.repeat(np.stack([v[c.bt[s, 0], 0] for s in range(len(ks))]), n, 0)).float().to(torch.bfloat16)
    assert not want.isnan().any() and (want.isinf().any() if n == 1 else want.isfinite().all())
    assert torch.equal(out, want)


def test_nan_reaches_only_what_attends_it():
    """A NaN value row (a key's, a whole block's by its scale) makes the rows that
    attend it NaN in its columns and leaves other sequences alone."""
    c = Case(28, 4, 128, 16, [1, 1, 1], [40, 40, 40], seed=3)
    ref, _ = c.run()
    c.v[c.bt[1, 1], 3, 2, 17] = 127
    c.s[c.bt[2, 1], 0, 1] = 255
    out, _ = c.run()
    assert torch.equal(out[0], ref[0])
    hit = out[1].isnan()
    assert hit[14:21, 17].all() and int(hit.sum()) == 7
    assert not out[2, 7:14].isfinite().any() and out[2, :7].isfinite().all() and out[2, 14:].isfinite().all()


def test_long_context_and_far_pages():
    """A 70,000-key sequence (several windows of its block table), and a pool
    whose pages lie beyond 2^32 bytes."""
    d, P, hkv = 128, 64, 4
    c = Case(28, hkv, d, P, [1, 3], [70_000, 30_000], seed=2)
    g = c.gpu()
    out = c.run("serial", g)
    c.check(*out, "long")
    used = c.k.shape[0]
    far = (5 << 30) // (P * hkv * d) + 1                   # first page past 5 GiB
    big = torch.zeros((far + used, P, hkv, d), dtype=torch.uint8, device="cuda")
    big[far:] = g["k"].view(torch.uint8)
    g["k"] = big.view(torch.float8_e4m3fn)
    vbig = torch.zeros_like(big)
    vbig[far:] = g["v"].view(torch.uint8)
    g["v"] = vbig.view(torch.float8_e4m3fn)
    s = torch.zeros((far + used, P // 16, hkv, 2), dtype=torch.uint8, device="cuda")
    s[far:] = g["s"].view(torch.uint8)
    g["s"] = s.view(torch.float8_e8m0fnu)
    g["bt"] = g["bt"] + far
    again = c.run("serial", g)
    assert torch.equal(again[0].view(torch.int16), out[0].view(torch.int16)) and torch.equal(again[1], out[1])


@pytest.mark.parametrize("hq,hkv,d,P,ns,ls", [
    (28, 4, 128, 16, [64], [4064]), (28, 4, 128, 64, [2, 20], [700, 1003]), (4, 1, 64, 16, [130, 1, 3], [1500, 40, 8300]),
    (32, 8, 64, 64, [33, 5], [900, 5]), (6, 3, 64, 64, [2], [385]), (16, 1, 128, 16, [300], [300]), (16, 1, 128, 16, [450], [450])])
def test_prefill_tiles_cut_along_their_keys(hq, hkv, d, P, ns, ls):
    """Few tiles: pieces of keys, whose rows may see none of a piece's, joined by a merge; other tiles stay whole
    (so do tiles of 448 keys or less, in two cases)."""
    log(f"kv8 cut prefill {hq}/{hkv} d{d} page {P} {ns} {ls}")
    c = Case(hq, hkv, d, P, ns, ls, seed=hq + P, spread=6)
    pa = c.plan()
    tiles = sum(-(-n * (hq // hkv) // 128) for n in ns if n > 1)
    assert (pa.plan.info["n_prefill_items"] > tiles) == (max(ls) > 448)
    out = c.run("prefill", pa=pa)
    single = torch.from_numpy(np.repeat(np.array(ns) == 1, ns))
    assert out[0][single].isnan().all()
    c.check(*c.run(pa=pa), "cut tiles")
    out = c.run(pa=pa, with_lse=False)
    c.check(out[0], None, "cut tiles, no log-sum-exp")


@pytest.mark.parametrize("hq,hkv,d,P,ns,ls,cut", [
    (28, 4, 128, 16, [85, 300, 85, 300, 85, 310], [2500, 3700, 2510, 3600, 85, 3711], False),
    (28, 4, 128, 16, [100] * 12, [3011 + 40 * k for k in range(12)], True), (32, 8, 64, 64, [300] * 4, [3100, 3001, 2999, 3200], True)])
def test_many_prefill_tiles_cut_along_their_keys(hq, hkv, d, P, ns, ls, cut):
    """More tiles than compute units, long ones: spread over all that is
    resident, but not where a few short ones are over."""
    c = Case(hq, hkv, d, P, ns, ls, seed=21)
    i, whole = c.plan().plan.info, sum(-(-n * (hq // hkv) // 128) for n in ns)
    assert whole * hkv > i["cus_prefill"] and (i["n_prefill_items"] > 1.5 * whole) == cut
    assert i["n_prefill_items"] * hkv <= 3 * i["cus_prefill"]
    c.check(*c.run(), "spread")


def test_cut_prefill_tiles_captured():
    c = Case(28, 4, 128, 16, [1, 40], [600, 1090], seed=12)
    g, pa = c.gpu(), c.plan()
    ref = c.run(g=g, pa=pa)
    out, lse = pa.alloc_out(g["q"], True)
    args = pa.kv8_args(g["q"], g["k"], g["v"], g["s"], g["bt"], g["ls"], g["qsl"], out, lse)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        F.flex_attn_mixed_kv8(pa.plan, args, F.FLEX_MODE_SERIAL)
    for k in range(3):
        out.zero_()
        lse.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.cpu().view(torch.int16), ref[0].view(torch.int16)) and torch.equal(lse.cpu(), ref[1]), f"replay {k}"
    c.check(*ref, "captured")


@pytest.mark.parametrize("hq,hkv,d,P", [(28, 4, 128, 16), (28, 4, 128, 64), (32, 8, 64, 16), (4, 4, 64, 64)])
def test_key_tiles_in_two_groups(hq, hkv, d, P):
    """Work-groups of two key groups: odd and even counts of key tiles, rows
    whose keys all lie in the first group's, a tile with nothing for the second."""
    ns, ls = [2, 3, 31, 33, 64, 100, 20, 2], [2, 40, 31, 97, 64, 290, 257, 33]
    c = Case(hq, hkv, d, P, ns, ls, seed=hq + d, spread=6)
    pa = c.plan(cus_decode=0)
    i = pa.plan.info
    assert i["n_prefill_items"] * i["prefill_grid_y"] <= i["cus_prefill"]
    c.check(*c.run("prefill", pa=pa), "two groups")


def test_prefill_crosses_a_block_table_window():
    """Page 16: 512 block-table entries cover 8192 keys; the chunk ends past that."""
    c = Case(4, 1, 64, 16, [70, 1], [8230, 9000], seed=9)
    c.check(*c.run(), "window")


@pytest.mark.parametrize("hq,hkv,d,P,n,L,whole", [
    (4, 1, 64, 16, 70, 8230, True), (4, 1, 64, 16, 30, 16500, False), (16, 1, 128, 16, 5, 8195, True), (16, 1, 128, 16, 40, 8200, True),
    (4, 1, 64, 64, 30, 16450, False), (4, 1, 64, 16, 30, 8230, True), (4, 1, 64, 64, 70, 16450, True)])
def test_whole_tiles_cross_block_table_windows(hq, hkv, d, P, n, L, whole):
    """512 entries of pages of 16, 256 of 64: tiles left whole (plans for one
    compute unit), by one key group and by two, end in a later window; long
    pieces of cut ones too."""
    c = Case(hq, hkv, d, P, [n], [L], seed=9)
    tiles = -(-n * (hq // hkv) // 128)
    pa = c.plan(cus_total=1)
    assert (pa.plan.info["n_prefill_items"] == tiles) == whole
    c.check(*c.run("prefill", pa=pa), "windows")


def test_strided_cache():
    """K and V interleaved in one pool with gaps, block-table rows wider than the plan's."""
    c = Case(28, 4, 128, 16, [1, 30, 1], [100, 60, 500], seed=8, width=3)
    g = c.gpu()
    ref = c.run(g=g)
    pages = c.k.shape[0]
    both = torch.full((pages, 2, c.P, c.hkv + 1, c.d + 16), 0x7F, dtype=torch.uint8, device="cuda")
    for i, n in enumerate("kv"):
        both[:, i, :, :c.hkv, :c.d] = g[n].view(torch.uint8)
        g[n] = both[:, i, :, :c.hkv, :c.d].view(torch.float8_e4m3fn)
    s = torch.full((pages, 3, 1, c.hkv, 2), 255, dtype=torch.uint8, device="cuda")
    s[:, 1] = g["s"].view(torch.uint8)
    g["s"] = s[:, 1].view(torch.float8_e8m0fnu)
    out = c.run(g=g)
    assert torch.equal(out[0].view(torch.int16), ref[0].view(torch.int16)) and torch.equal(out[1], ref[1])
    c.check(*out, "strided")


@pytest.mark.parametrize("hq,hkv,d,P", [(28, 4, 128, 16), (20, 20, 64, 64), (24, 12, 128, 64), (4, 1, 64, 16)])
def test_sequences_of_many_pieces(hq, hkv, d, P):
    """More than eight pieces a sequence in the mean: merged a row at a time,
    the rows of the heads that exist only (20 and 12 KV heads in columns of 8)."""
    c = Case(hq, hkv, d, P, [1, 1, 1], [5000, 2999, 64], seed=hq)
    pa = c.plan()
    assert pa.plan.info["n_decode_items"] > 8 * pa.plan.info["n_split_seqs"]
    c.check(*c.run("decode", pa=pa), "many pieces")


@pytest.mark.parametrize("hq,hkv,d,P", [(28, 4, 128, 16), (10, 5, 64, 16), (8, 8, 64, 64), (4, 1, 64, 64)])
def test_head_major_pages(hq, hkv, d, P):
    """Pages laid out [head][slot][dim]: the rows behind a head's last key are
    the next head's, and hold NaN in the last page."""
    c = Case(hq, hkv, d, P, [1, 30, 1, 1], [100, 60, 500, 5], seed=hq)
    g = c.gpu()
    ref = c.run(g=g, min_split_tokens=64)
    for n in "kv":
        g[n] = g[n].view(torch.uint8).transpose(1, 2).contiguous().transpose(1, 2).view(torch.float8_e4m3fn)
    out = c.run(g=g, min_split_tokens=64)
    assert torch.equal(out[0].view(torch.int16), ref[0].view(torch.int16)) and torch.equal(out[1], ref[1])
    c.check(*out, "head major")


def test_captured_and_on_two_streams():
    c = Case(28, 4, 128, 16, [1, 1, 40], [3000, 500, 90], seed=10)
    ref = c.run(min_split_tokens=64)
    g, pa = c.gpu(), c.plan(min_split_tokens=64)
    out, lse = pa.alloc_out(g["q"], True)
    args = pa.kv8_args(g["q"], g["k"], g["v"], g["s"], g["bt"], g["ls"], g["qsl"], out, lse)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        F.flex_attn_mixed_kv8(pa.plan, args, F.FLEX_MODE_SERIAL)
    for k in range(3):
        out.zero_()
        lse.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.cpu().view(torch.int16), ref[0].view(torch.int16)) and torch.equal(lse.cpu(), ref[1]), f"replay {k}"
    # two runs in flight, each with a workspace of its own
    streams, runs = [torch.cuda.Stream() for _ in range(2)], []
    for s in streams:
        p2 = c.plan(min_split_tokens=64)
        o, e = p2.alloc_out(g["q"], True)
        runs.append((p2, o, e, p2.kv8_args(g["q"], g["k"], g["v"], g["s"], g["bt"], g["ls"], g["qsl"], o, e)))
    torch.cuda.synchronize()
    for s, (p2, o, e, a2) in zip(streams, runs):
        F.flex_attn_mixed_kv8(p2.plan, a2, F.FLEX_MODE_SERIAL, stream=s.cuda_stream)
    torch.cuda.synchronize()
    for _, o, e, _ in runs:
        assert torch.equal(o.cpu().view(torch.int16), ref[0].view(torch.int16)) and torch.equal(e.cpu(), ref[1])


def test_debug_mode_checks_the_run():
    c = Case(28, 4, 128, 16, [1, 3], [40, 20], seed=1)
    prev = F.set_debug(1)
    try:
        c.check(*c.run(), "debug")
        g = c.gpu()
        g["bt"][1, 1] = c.k.shape[0]
        with pytest.raises(F.FlexAttnError) as e:
            c.run(g=g)
        assert e.value.status == F.FLEX_ERR_INVALID_ARG and "sequence 1" in str(e.value)
    finally:
        F.set_debug(prev)


def test_steps_of_append_and_attention():
    """As a serving loop uses them: prompts arrive, then decode, four steps of
    rotation, append and attention over one 8-bit cache; every step's outputs
    against attention over the values the oracle's append holds."""
    hq, hkv, d, P, B = 28, 4, 128, 16, 3
    bt, _, _, pages = batch([0] * B, [80] * B, P, 5)
    kc, vc, sc = F.make_kv8_cache(pages, P, hkv, d)
    host = [x.view(torch.uint8).cpu().numpy().copy() for x in (kc, vc, sc)]
    shape = F.make_shape(hq, hkv, d, d, P, scale_of(d))
    tab = F.rope_table(256, d)
    d_bt = torch.from_numpy(bt).cuda()
    have = [0] * B
    for step, ns in enumerate([[37, 50, 0], [1, 1, 20], [1, 1, 9], [1, 1, 1]]):
        have = [h + n for h, n in zip(have, ns)]
        ls, qsl = np.array(have, dtype=np.int32), np.concatenate([[0], np.cumsum(ns)]).astype(np.int32)
        T = int(qsl[-1])
        rows = bf16((T, hq + 2 * hkv, d), 100 + step, 1.5)
        row = rows.cuda()
        q_out = torch.empty((T, hq, d), dtype=torch.bfloat16, device="cuda")
        d_ls, d_qsl = torch.from_numpy(ls).cuda(), torch.from_numpy(qsl).cuda()
        F.flex_attn_kv8_append(shape, F.make_rope(tab), F.make_kv8_append_args(
            row[:, hq:hq + hkv], row[:, hq + hkv:], d_bt, d_ls, d_qsl, kc, vc, sc, row[:, :hq], q_out))
        pa = F.PagedAttention(shape, F.make_opts(kv_bits=8), qsl, ls, bt.shape[1])
        out, lse = pa.alloc_out(q_out, True)
        args = pa.kv8_args(q_out, kc, vc, sc, d_bt, d_ls, d_qsl, out, lse)
        F.flex_attn_mixed_kv8(pa.plan, args, F.FLEX_MODE_SERIAL)
        torch.cuda.synchronize()
        pos = np.concatenate([np.arange(L - n, L) for n, L in zip(ns, ls)])[None]
        turned = RK.rotate(rows[:, hq:hq + hkv].float().numpy(), tab.cpu().numpy(), pos, dtype=np.float32)
        host[0], ks = RK.kv8_append(host[0], host[2][..., 0], turned, bt, ls, qsl, P)
        host[1], vs = RK.kv8_append(host[1], host[2][..., 1], rows[:, hq + hkv:].float().numpy(), bt, ls, qsl, P)
        host[2] = np.stack([ks, vs], -1)
        for got, want in zip((kc, vc, sc), host):
            assert np.array_equal(got.view(torch.uint8).cpu().numpy(), want), f"step {step}: the cache"
        vals = RK.values(host[0], host[2][..., 0]), RK.values(host[1], host[2][..., 1])
        ref = attend64(q_out.cpu(), *vals, bt, ls, qsl, np.float64(np.float32(scale_of(d))))
        check_attention(out.cpu(), lse.cpu(), ref, ls, qsl, d, f"step {step}")
