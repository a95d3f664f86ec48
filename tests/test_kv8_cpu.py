"""Rotary positions and the 8-bit cache on the CPU: pins of their oracle,
refusals of the C calls and of the binding, and plans for 8-bit caches."""
import ctypes
import math
import pathlib
import random

import numpy as np
import pytest
import torch

import oracle.rope_kv8 as RK
from oracle import plan as OP
from paper_2606_04415_amd import flexattn as F

from kv8_common import batch, bf16, cache8
from test_abi_cpu import compare


# ---- the oracle ----

def test_codes_are_torchs():
    """Every code's value and the rounding of a sweep of values are torch's e4m3fn."""
    every = torch.arange(256, dtype=torch.int32).to(torch.uint8)
    v = every.view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(np.nan_to_num(v, nan=999.0), np.nan_to_num(RK.VALUES, nan=999.0))
    x = np.concatenate([np.linspace(-448, 448, 200_001), np.geomspace(2.0 ** -14, 448, 100_001)]).astype(np.float32)
    mid = (RK.VALUES[:126] + RK.VALUES[1:127]) / 2                     # ties
    x = np.concatenate([x, mid.astype(np.float32), -mid.astype(np.float32)])
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    got = RK.encode(x)
    assert np.array_equal(RK.VALUES[got], RK.VALUES[want])


def test_rotation_is_a_complex_product_and_keeps_differences():
    x = np.random.RandomState(0).randn(5, 3, 32)
    tab = F.rope_table(100, 32, device="cpu").double().numpy()
    pos = np.array([[3, 0, 99, 50, 7]])
    z = x[..., :16] + 1j * x[..., 16:]
    w = z * (tab[pos[0], :16] + 1j * tab[pos[0], 16:])[:, None]
    assert np.allclose(RK.rotate(x, tab, pos), np.concatenate([w.real, w.imag], -1), rtol=0, atol=1e-12)
    y = RK.rotate(x, tab, pos, neighbours=True)
    z = (x[..., 0::2] + 1j * x[..., 1::2]) * (tab[pos[0], :16] + 1j * tab[pos[0], 16:])[:, None]
    assert np.allclose(y[..., 0::2], z.real) and np.allclose(y[..., 1::2], z.imag)
    # scores depend on the distance alone
    q, k = np.random.RandomState(1).randn(2, 1, 1, 32)
    def score(a, b):
        return (RK.rotate(q, tab, np.array([[a]])) * RK.rotate(k, tab, np.array([[b]]))).sum()
    assert abs(score(60, 40) - score(25, 5)) < 1e-5


def test_axes_of_pairs():
    assert RK.axis_of_pairs(8, [2, 3, 3], False) == [0, 0, 1, 1, 1, 2, 2, 2]
    assert RK.axis_of_pairs(8, [4, 2, 2], True) == [0, 1, 2, 0, 1, 2, 0, 0]
    for s, dealt in (([24, 20, 20], True), ([16, 24, 24], False), ([1, 0, 63], False)):
        a = RK.axis_of_pairs(64, s, dealt)
        assert [a.count(i) for i in range(3)] == s


def test_rope_table_is_exact_at_far_positions():
    t = F.rope_table(1 << 17, 16, 1e6, device="cpu").double()
    for p in (0, 1, 4097, (1 << 17) - 1):
        for i in range(8):
            a = p * 1e6 ** (-i / 8)
            assert abs(float(t[p, i]) - math.cos(a)) <= 2.0 ** -24 and abs(float(t[p, 8 + i]) - math.sin(a)) <= 2.0 ** -24


def test_append_token_by_token_bounds_the_error():
    """Whatever the order of sizes, a cached value is off by at most half a step
    of its code at each scale its block had: 2^-4 of the value, or half the
    smallest code (2^-10) times the largest scale, per coding."""
    r = np.random.RandomState(3)
    codes, scales = np.zeros((2, 16, 1, 8), dtype=np.uint8), np.zeros((2, 1, 1), dtype=np.uint8)
    bt = np.array([[1, 0]], dtype=np.int32)
    rows = (r.randn(20, 1, 8) * np.exp(3 * r.randn(20, 1, 1))).astype(np.float32)
    for t in range(20):
        before = scales.copy()
        codes, scales = RK.kv8_append(codes, scales, rows[t:t + 1], bt, [t + 1], [0, 1], 16)
        page = bt[0, t // 16]
        assert t % 16 == 0 or scales[page, 0, 0] >= before[page, 0, 0]
        assert np.abs(rows[t]).max() <= 448 * 2.0 ** (int(scales[page, 0, 0]) - 127)
    v = RK.values(codes, scales)
    for t in range(20):
        page = bt[0, t // 16]
        top = 2.0 ** (int(scales[page, 0, 0]) - 127)
        # rounded once normally; below 2^-6 of the scale once more for every growth, each half a step of 2^-9
        assert (np.abs(v[page, t % 16] - rows[t]) <= np.abs(rows[t]) * 2.0 ** -4 + 2.0 ** -9 * top).all()


def test_a_scale_too_small_by_one_is_caught():
    """The oracle's own check of what a wrong border would do: 450 does not fit 448."""
    assert RK.scale_exponent(448.0) == 0 and RK.scale_exponent(448.0001) == 1 and RK.scale_exponent(0.0) == -117
    assert RK.scale_exponent(224.0) == -1 and RK.scale_exponent(2.0 ** 127) == 119


# ---- plans ----

GQA = [OP.Shape(28, 4, 128, 128, 16, 128 ** -0.5, 0), OP.Shape(4, 1, 64, 64, 16, 0.125, 0),
       OP.Shape(32, 2, 128, 128, 64, 0.1, 0), OP.Shape(64, 8, 128, 128, 16, 0.088, 0), OP.Shape(20, 20, 64, 64, 64, 0.1, 0)]


def test_plans_for_8_bit_caches_match_the_rederivation():
    rng = random.Random(2)
    for _ in range(150):
        sh = rng.choice(GQA)
        ns, ls = [], []
        for _ in range(rng.randint(0, 40)):
            L = rng.choice([0, 1, 15, 16, 17, 129, 4095, rng.randint(1, 20000)])
            ns.append(0 if L == 0 else 1 if rng.random() < 0.6 else rng.randint(0, L))
            ls.append(L)
        qsl = np.concatenate([[0], np.cumsum(ns)]).astype(int).tolist()
        maxp = max([1] + [-(-L // sh.page_size) for L in ls])
        compare(sh, OP.Opts(kv_bits=8, cus_decode=rng.choice([0, 96, -1]), min_split_tokens=rng.choice([0, 16]),
                            bm=rng.choice([0, 128]), decode_tail=rng.choice([0, -1])), qsl, ls, maxp)


@pytest.mark.parametrize("count,top,whole", [(1, 128, True), (1, 129, False), (9, 2, True), (15, 129, False), (16, 256, True), (16, 257, False),
                                             (700, 250, True), (3000, 5, True), (300, 3000, False)])
@pytest.mark.parametrize("co", [0, 96])
def test_short_decode_sequences_stay_whole(count, top, whole, co):
    """Ranges of whole sequences by default, beside a prefill too; by pages when
    the caller sets the least range; no range shorter than the mean sequence."""
    rng = random.Random(count * top)
    ls = [top] + [rng.randint(1, top) for _ in range(count - 1)]
    ns = [1] * count + ([40] if co else [])
    ls += [40] if co else []
    qsl = np.concatenate([[0], np.cumsum(ns)]).astype(int).tolist()
    for sh in GQA:
        maxp = max(-(-x // sh.page_size) for x in ls)
        shape = F.make_shape(sh.num_q_heads, sh.num_kv_heads, sh.head_dim_qk, sh.head_dim_v, sh.page_size, sh.sm_scale)
        for kw in ({}, dict(min_split_tokens=64)):
            compare(sh, OP.Opts(kv_bits=8, cus_decode=co, decode_tail=-1 if co else 0, **kw), qsl, ls, maxp)
        i = F.flex_attn_plan(shape, F.make_opts(kv_bits=8, cus_decode=co, decode_tail=-1 if co else 0), qsl, ls, maxp).info
        assert (i["n_split_seqs"] == 0 and i["n_decode_items"] == count) or not whole
        assert not whole or i["n_decode_ranges"] == min(count, (co or 256) // i["decode_wg_width"])
        assert i["n_decode_ranges"] <= max(count, sum(-(-x // sh.page_size) for x in ls[:count]) * sh.page_size // 64)


@pytest.mark.parametrize("n,ls,cut", [((64,), (4000,), True), ((2,), (300,), False), ((2,), (448,), False), ((2,), (449,), True), ((64, 3), (64, 2500), True),
                                      ((64, 1, 200), (4000, 900, 210), True), ((3000,), (3000,), False), ((200,) * 5, (3000,) * 5, False),
                                      ((170,) * 7, (6170,) * 7, True), ((1200,), (5200,), True), ((2048,), (2048,), False)])
def test_few_prefill_tiles_are_cut_along_their_keys(n, ls, cut):
    """Pieces of a tile are disjoint, in order and cover its keys; slots are
    those of the workspace, one after another; work-groups stay within the units."""
    sh = GQA[0]
    qsl = np.concatenate([[0], np.cumsum(n)]).astype(int).tolist()
    maxp = max(-(-x // sh.page_size) for x in ls)
    compare(sh, OP.Opts(kv_bits=8), qsl, list(ls), maxp)
    p = F.flex_attn_plan(F.make_shape(sh.num_q_heads, sh.num_kv_heads, sh.head_dim_qk, sh.head_dim_v, sh.page_size, sh.sm_scale),
                         F.make_opts(kv_bits=8), qsl, list(ls), maxp)
    info, w = p.info, list(p.export())
    items = [w[w[10] + 8 * i:w[10] + 8 * i + 8] for i in range(info["n_prefill_items"])]   # w[10]: where they start
    pieces = [it for it in items if it[6] > 1]
    assert bool(pieces) == cut
    if not cut:
        return
    slots = info["cus_prefill"] * (1 if 2 * sum(-(-x * 7 // 128) for x in n if x > 1) * 4 <= info["cus_prefill"] else 3)
    assert info["workspace_bytes"] > 0 and len(items) * info["prefill_grid_y"] <= slots
    for tile in {tuple(it[:4]) for it in pieces}:
        own = sorted((it for it in pieces if tuple(it[:4]) == tile), key=lambda it: it[5])
        s, _, _, r1 = tile
        assert own[0][5] == 0 and own[-1][4] == ls[s] - n[s] + (r1 - 1) // 7 + 1 and own[0][6] == len(own)
        assert all(a[4] == b[5] and a[4] % 64 == 0 and a[7] + 1 == b[7] for a, b in zip(own, own[1:]))
    assert sorted(it[7] for it in pieces) == list(range(len(pieces)))


@pytest.mark.parametrize("sh,opts", [
    (GQA[0], OP.Opts(kv_bits=4)), (GQA[0], OP.Opts(kv_bits=-8)), (GQA[0], OP.Opts(kv_bits=8, bm=32)),
    (GQA[0], OP.Opts(kv_bits=8, bm=16)), (OP.Shape(128, 1, 576, 512, 64, 0.07, 1), OP.Opts(kv_bits=8)),
    (OP.Shape(16, 16, 192, 128, 64, 0.07, 0), OP.Opts(kv_bits=8)), (GQA[0], OP.Opts(kv_bits=16)),
])
def test_plan_options_status(sh, opts):
    compare(sh, opts, [0, 1, 3], [5, 9], 4)


def test_decode_bytes_count_codes_and_scales():
    p = F.flex_attn_plan(F.make_shape(28, 4, 128, 128, 16, 0.1), F.make_opts(kv_bits=8), [0, 1, 2], [100, 16], 8)
    assert p.info["decode_bytes"] == 116 * 4 * 256 + (7 + 1) * 4 * 2 and p.info["n_fused_wgs"] == 0 and p.info["bm"] == 128


# ---- refusals of the C calls (no GPU is touched) ----

FAKE = 0x10000


def rope(**kw):
    r = F.Rope()
    r.cos_sin, r.positions, r.positions_stride, r.max_position = FAKE, FAKE, 100, 64
    r.rot_begin, r.rot_dim, r.neighbours, r.n_axes, r.dealt = 0, 128, 0, 1, 0
    for k, v in kw.items():
        setattr(r, k, (ctypes.c_int32 * 4)(*v) if k == "sections" else v)
    return r


SHAPE = F.make_shape(28, 4, 128, 128, 16, 0.1)
ROW = (ctypes.c_int64 * 3)(16 * 4 * 128, 4 * 128, 128)


def rope_args(n=10, **kw):
    a = F.RopeAppendArgs()
    a.kv.k_new, a.kv.v_new, a.kv.slot_mapping, a.kv.k_cache, a.kv.v_cache = FAKE, FAKE, FAKE, FAKE, FAKE
    a.kv.k_new_stride = a.kv.v_new_stride = 512
    a.kv.n_tokens, a.kv.num_pages, a.kv.k_stride, a.kv.v_stride = n, 4, ROW, ROW
    a.q, a.q_stride, a.q_out = FAKE, 28 * 128, 0x4000000
    for k, v in kw.items():
        setattr(a.kv if hasattr(a.kv, k) else a, k, v)
    return a


def kv8_append_args(n=10, **kw):
    a = F.Kv8AppendArgs()
    for f in ("k_new", "v_new", "q", "block_table", "seq_lens", "query_start_loc", "k_cache", "v_cache", "kv_scales"):
        setattr(a, f, FAKE)
    a.k_new_stride = a.v_new_stride = 512
    a.q_stride, a.q_out = 28 * 128, 0x4000000
    a.n_tokens, a.num_seqs, a.block_table_stride, a.num_pages = n, 2, 4, 4
    a.k_stride = a.v_stride = ROW
    a.scale_page_stride = 8
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def refused(fn, *args, status=F.FLEX_ERR_INVALID_ARG):
    st = getattr(F.lib(), fn)(*args, None)
    assert st == status, (st, F.last_error())
    return F.last_error()


@pytest.mark.parametrize("kw", [
    dict(cos_sin=None), dict(cos_sin=FAKE + 4), dict(max_position=0), dict(rot_dim=0), dict(rot_dim=24), dict(rot_dim=144),
    dict(rot_begin=4), dict(rot_begin=-8), dict(rot_begin=8), dict(rot_begin=2 ** 31 - 8), dict(n_axes=0), dict(n_axes=5),
    dict(neighbours=2), dict(dealt=-1), dict(positions=None), dict(n_axes=3, sections=[16, 24, 23]),
    dict(n_axes=3, sections=[16, 49, -1]), dict(n_axes=2, sections=[65, -1]), dict(n_axes=3, sections=[16, 24, 24], positions_stride=9),
    dict(n_axes=3, sections=[20, 22, 22], dealt=1), dict(n_axes=2, sections=[2 ** 31 - 1, 65]),
])
def test_rope_refusals(kw):
    refused("flex_attn_rope_append", ctypes.byref(SHAPE), ctypes.byref(rope(**kw)), ctypes.byref(rope_args()))
    if kw != dict(positions=None):
        refused("flex_attn_kv8_append", ctypes.byref(SHAPE), ctypes.byref(rope(**kw)), ctypes.byref(kv8_append_args()))


def test_kv8_append_needs_positions_for_several_axes():
    r = rope(positions=None, n_axes=2, sections=[32, 32])
    assert "positions" in refused("flex_attn_kv8_append", ctypes.byref(SHAPE), ctypes.byref(r), ctypes.byref(kv8_append_args()))


@pytest.mark.parametrize("kw", [
    dict(n_tokens=-1), dict(k_new=None), dict(v_new=None), dict(slot_mapping=None), dict(k_cache=None), dict(q=None),
    dict(q_out=None), dict(q=FAKE + 8), dict(q_out=FAKE + 2), dict(q_stride=28 * 128 - 8), dict(q_stride=28 * 128 + 4),
    dict(k_new_stride=504), dict(num_pages=0), dict(q_out=FAKE + 256), dict(q_stride=28 * 128 + 8, q_out=FAKE),
    dict(k_stride=(ctypes.c_int64 * 3)(8192, 512, 64)), dict(k_stride=(ctypes.c_int64 * 3)(8192, 516, 128)),
])
def test_rope_append_refusals(kw):
    refused("flex_attn_rope_append", ctypes.byref(SHAPE), ctypes.byref(rope()), ctypes.byref(rope_args(**kw)))


def test_append_null_and_shape_refusals():
    r, a, b = rope(), rope_args(), kv8_append_args()
    refused("flex_attn_rope_append", None, ctypes.byref(r), ctypes.byref(a))
    refused("flex_attn_rope_append", ctypes.byref(SHAPE), None, ctypes.byref(a))
    refused("flex_attn_rope_append", ctypes.byref(SHAPE), ctypes.byref(r), None)
    refused("flex_attn_kv8_append", None, None, ctypes.byref(b))
    refused("flex_attn_kv8_append", ctypes.byref(SHAPE), None, None)
    odd = F.make_shape(28, 4, 96, 96, 16, 0.1)
    refused("flex_attn_rope_append", ctypes.byref(odd), ctypes.byref(r), ctypes.byref(a), status=F.FLEX_ERR_UNSUPPORTED)
    for sh in (F.make_shape(128, 1, 576, 512, 64, 0.1, True), F.make_shape(16, 16, 192, 128, 64, 0.1)):
        refused("flex_attn_kv8_append", ctypes.byref(sh), None, ctypes.byref(b), status=F.FLEX_ERR_UNSUPPORTED)
    # nothing to do: nothing is launched, nor asked of the pointers
    for fn, x in (("flex_attn_rope_append", F.RopeAppendArgs()), ("flex_attn_kv8_append", F.Kv8AppendArgs())):
        assert getattr(F.lib(), fn)(ctypes.byref(SHAPE), ctypes.byref(r), ctypes.byref(x), None) == F.FLEX_OK


@pytest.mark.parametrize("kw", [
    dict(n_tokens=-1), dict(num_seqs=-1), dict(k_new=None), dict(v_new=None), dict(block_table=None), dict(seq_lens=None),
    dict(query_start_loc=None), dict(k_cache=None), dict(v_cache=None), dict(kv_scales=None), dict(kv_scales=FAKE + 1),
    dict(scale_page_stride=6), dict(scale_page_stride=9), dict(scale_page_stride=2 ** 31), dict(block_table_stride=0),
    dict(num_pages=0), dict(k_new_stride=511), dict(v_new=FAKE + 8), dict(v_cache=FAKE + 8), dict(v_new_stride=500),
    dict(k_stride=(ctypes.c_int64 * 3)(8192, 512, 112)), dict(v_stride=(ctypes.c_int64 * 3)(8192, 520, 128)),
    dict(k_stride=(ctypes.c_int64 * 3)(0, 512, 128)), dict(q=None), dict(q_out=None), dict(q_out=FAKE + 16),
])
def test_kv8_append_refusals(kw):
    refused("flex_attn_kv8_append", ctypes.byref(SHAPE), ctypes.byref(rope()), ctypes.byref(kv8_append_args(**kw)))


def run_args(plan):
    a = F.Kv8Args()
    x = a.attn
    x.q = x.k_cache = x.v_cache = x.block_table = x.seq_lens = x.query_start_loc = x.out = x.d_plan = x.workspace = FAKE
    x.k_stride, x.v_stride = ROW, ROW
    x.num_pages, x.block_table_stride, x.d_plan_bytes, x.workspace_bytes = 10, 4, plan.info["device_plan_bytes"], 1 << 30
    a.kv_scales, a.scale_page_stride = FAKE, 8
    return a


def test_attention_refusals():
    plan = F.flex_attn_plan(SHAPE, F.make_opts(kv_bits=8, min_split_tokens=16), [0, 1, 3], [40, 50], 4)
    wide = F.flex_attn_plan(SHAPE, F.make_opts(min_split_tokens=16), [0, 1, 3], [40, 50], 4)

    def every(a, p=plan, mode=F.FLEX_MODE_SERIAL, status=F.FLEX_ERR_INVALID_ARG):
        x = ctypes.byref(a) if a is not None else None
        for fn in (F.lib().flex_attn_decode_kv8, F.lib().flex_attn_prefill_kv8):
            assert fn(p.handle if p else None, x, None) == status, F.last_error()
        assert F.lib().flex_attn_mixed_kv8(p.handle if p else None, x, mode, None, None) == status, F.last_error()
        return F.last_error()

    every(None)
    every(run_args(plan), p=None)
    assert "kv_bits" in every(run_args(plan), p=wide)
    for f, v in (("kv_scales", None), ("kv_scales", FAKE + 1), ("scale_page_stride", 6), ("scale_page_stride", 11)):
        a = run_args(plan)
        setattr(a, f, v)
        assert "scale" in every(a)
    for f, v in (("q", None), ("q", FAKE + 4), ("k_cache", FAKE + 8), ("v_cache", None), ("num_pages", 0), ("block_table_stride", 3),
                 ("k_stride", (ctypes.c_int64 * 3)(8192, 520, 128)), ("v_stride", (ctypes.c_int64 * 3)(8192, 512, 64)),
                 ("k_stride", (ctypes.c_int64 * 3)(1 << 31, 512, 128)), ("v_stride", (ctypes.c_int64 * 3)(8192, 1 << 27, 128)),
                 ("k_stride", (ctypes.c_int64 * 3)(8192, 512, 1 << 31)), ("workspace", None)):
        a = run_args(plan)
        setattr(a.attn, f, v)
        every(a)
    a = run_args(plan)
    a.attn.workspace_bytes = 16
    every(a, status=F.FLEX_ERR_WORKSPACE)
    a = run_args(plan)
    a.attn.d_plan_bytes = 8
    every(a, status=F.FLEX_ERR_WORKSPACE)
    x = ctypes.byref(run_args(plan))
    assert F.lib().flex_attn_mixed_kv8(plan.handle, x, 9, None, None) == F.FLEX_ERR_INVALID_ARG
    assert F.lib().flex_attn_mixed_kv8(plan.handle, x, F.FLEX_MODE_FUSED, None, None) == F.FLEX_ERR_UNSUPPORTED
    assert F.lib().flex_attn_mixed_kv8(plan.handle, x, F.FLEX_MODE_CORUN, None, None) == F.FLEX_ERR_INVALID_ARG
    # and the bf16 calls refuse a plan for an 8-bit cache
    b = ctypes.byref(run_args(plan).attn)
    for fn in (F.lib().flex_attn_decode, F.lib().flex_attn_prefill):
        assert fn(plan.handle, b, None) == F.FLEX_ERR_INVALID_ARG
    for fn in (F.lib().flex_attn_mixed, F.lib().flex_attn_mixed_static):
        assert fn(plan.handle, b, F.FLEX_MODE_SERIAL, None, None) == F.FLEX_ERR_INVALID_ARG
    assert F.lib().flex_attn_debug_gather(plan.handle, b, 0, 40, FAKE, FAKE, None) == F.FLEX_ERR_UNSUPPORTED


# ---- refusals of the binding ----

def tensors():
    bt, ls, qsl, pages = batch([1, 2], [40, 20], 16, 1)
    k, v, s = (torch.from_numpy(x) for x in cache8(pages, 16, 4, 128, 1))
    return dict(q=bf16((3, 28, 128), 1), k_new=bf16((3, 4, 128), 2), v_new=bf16((3, 4, 128), 3), bt=torch.from_numpy(bt),
                ls=torch.from_numpy(ls), qsl=torch.from_numpy(qsl), k=k.view(torch.float8_e4m3fn), v=v.view(torch.float8_e4m3fn),
                s=s.view(torch.float8_e8m0fnu), q_out=torch.empty(3, 28, 128, dtype=torch.bfloat16),
                out=torch.empty(3, 28, 128, dtype=torch.bfloat16))


def kv8_append(t, shape=SHAPE, rope=None, **kw):
    t = dict(t, **kw)
    a = F.make_kv8_append_args(t["k_new"], t["v_new"], t["bt"], t["ls"], t["qsl"], t["k"], t["v"], t["s"], t["q"], t["q_out"])
    F.flex_attn_kv8_append(shape, rope, a)


@pytest.mark.parametrize("name,change,match", [
    ("k", lambda x: x.view(torch.uint8), "float8_e4m3fn"), ("s", lambda x: x.view(torch.uint8), "float8_e8m0fnu"),
    ("s", lambda x: x[:-1], "kv_scales"), ("s", lambda x: x.view(torch.uint8).transpose(2, 3).contiguous().transpose(2, 3).view(x.dtype), "contiguous"),
    ("v", lambda x: x[:, :, :2], "v_cache|same shape"), ("k_new", lambda x: x.float(), "bfloat16"), ("k_new", lambda x: x[:2], "same tokens"),
    ("v_new", lambda x: x.transpose(1, 2).contiguous().transpose(1, 2), "contiguous rows"), ("bt", lambda x: x.long(), "block_table"),
    ("bt", lambda x: x[:1], "block_table"), ("ls", lambda x: x.long(), "int32"), ("qsl", lambda x: x[:2], "query_start_loc"),
    ("q", lambda x: x[:2], "q_out|same tokens"), ("q_out", lambda x: None, "together"), ("q_out", lambda x: x.float(), "q_out"),
])
def test_binding_refuses_append_tensors(name, change, match):
    t = tensors()
    with pytest.raises(ValueError, match=match):
        kv8_append(t, **{name: change(t[name])})


def test_binding_refuses_cpu_tensors_and_other_shapes():
    t = tensors()
    with pytest.raises(ValueError, match="GPU tensors"):
        kv8_append(t)
    with pytest.raises(ValueError, match="shape"):
        kv8_append(t, shape=F.make_shape(28, 4, 128, 128, 64, 0.1))
    with pytest.raises(ValueError, match="shape"):
        kv8_append(t, shape=F.make_shape(32, 4, 128, 128, 16, 0.1))
    a = F.make_kv8_args(t["q"], t["k"], t["v"], t["s"], t["bt"], t["ls"], t["qsl"], t["out"])
    plan = F.flex_attn_plan(SHAPE, F.make_opts(kv_bits=8), [0, 1, 3], [40, 20], 3)
    for call in (lambda: F.flex_attn_decode_kv8(plan, a), lambda: F.flex_attn_prefill_kv8(plan, a),
                 lambda: F.flex_attn_mixed_kv8(plan, a, F.FLEX_MODE_SERIAL)):
        with pytest.raises(ValueError, match="GPU tensors"):
            call()
    for p, match in ((F.flex_attn_plan(F.make_shape(28, 4, 128, 128, 64, 0.1), F.make_opts(kv_bits=8), [0, 1, 3], [40, 20], 3), "shape"),
                     (F.flex_attn_plan(SHAPE, F.make_opts(kv_bits=8), [0, 1], [40], 3), "1 and 1"),
                     (F.flex_attn_plan(SHAPE, F.make_opts(kv_bits=8), [0, 1, 4], [40, 20], 3), "2 and 4")):
        for call in (lambda: F.flex_attn_decode_kv8(p, a), lambda: F.flex_attn_prefill_kv8(p, a),
                     lambda: F.flex_attn_mixed_kv8(p, a, F.FLEX_MODE_SERIAL)):
            with pytest.raises(ValueError, match=match):
                call()
    kc = torch.zeros(4, 16, 4, 128, dtype=torch.bfloat16)
    slots, tab = torch.arange(3, dtype=torch.int32), F.rope_table(64, 128, device="cpu")
    pos = torch.zeros(3, dtype=torch.int32)
    b = F.make_rope_append_args(t["q"], t["q_out"], t["k_new"], t["v_new"], slots, kc, kc.clone())
    with pytest.raises(ValueError, match="GPU tensors"):
        F.flex_attn_rope_append(SHAPE, F.make_rope(tab, pos), b)
    with pytest.raises(ValueError, match="2 positions"):
        F.flex_attn_rope_append(SHAPE, F.make_rope(tab, pos[:2]), b)
    with pytest.raises(ValueError, match="sections"):
        F.make_rope(tab, pos[None].expand(3, 3))
    with pytest.raises(ValueError, match="float32"):
        F.make_rope(tab.double(), pos)
    with pytest.raises(ValueError, match="int32"):
        F.make_rope(tab, pos.long())
    with pytest.raises(ValueError, match="slot_mapping"):
        F.make_rope_append_args(t["q"], t["q_out"], t["k_new"], t["v_new"], slots[:2], kc, kc.clone())
    with pytest.raises(ValueError, match="bfloat16"):
        F.make_kv8_args(t["q"].float(), t["k"], t["v"], t["s"], t["bt"], t["ls"], t["qsl"], t["out"])
    with pytest.raises(ValueError, match="out must"):
        F.make_kv8_args(t["q"], t["k"], t["v"], t["s"], t["bt"], t["ls"], t["qsl"], t["out"][:2])
    with pytest.raises(ValueError, match="lse must"):
        F.make_kv8_args(t["q"], t["k"], t["v"], t["s"], t["bt"], t["ls"], t["qsl"], t["out"], torch.zeros(3, 27))
    with pytest.raises(ValueError, match="as many sequences"):
        F.make_kv8_args(t["q"], t["k"], t["v"], t["s"], t["bt"], t["ls"], t["qsl"][:2], t["out"])


@pytest.mark.parametrize("kv_bits", [8, 16])
def test_a_plan_that_does_not_fit_the_host_is_an_error(kv_bits):
    """A prompt whose tiles take gigabytes, in a process that may have a quarter of
    one more: a status, not an exception through the C call, which would end the
    process; and the next plan is made."""
    import subprocess
    import sys
    code = f"""
import resource
from paper_2606_04415_amd import flexattn as F
shape = F.make_shape(28, 4, 128, 128, 16, 0.1)
opts = F.make_opts(kv_bits={kv_bits}, bm=128)
F.flex_attn_plan(shape, opts, [0, 1], [5], 1)
held = next(int(x.split()[1]) for x in open("/proc/self/status") if x.startswith("VmSize")) * 1024
resource.setrlimit(resource.RLIMIT_AS, (held + (256 << 20), resource.RLIM_INFINITY))
n = 300_000_000
try:
    F.flex_attn_plan(shape, opts, [0, n], [n], n // 16)
    print("made")
except F.FlexAttnError as e:
    print("status", e.status, F.flex_attn_plan(shape, opts, [0, 40], [50], 4).info["n_prefill_items"] > 0)
"""
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=120,
                       cwd=pathlib.Path(__file__).resolve().parents[1])
    assert r.stdout.split() == ["status", str(F.FLEX_ERR_INTERNAL), "True"], (r.returncode, r.stdout, r.stderr[-500:])


def test_plans_take_the_starts_that_the_batch_needs():
    """query_start_loc may go on past the batch (a buffer of the largest one), be a
    column, or be empty for an empty batch, as before plans knew their batch."""
    for qsl, ls in (([0, 1, 4, 0, 0], [9, 8]), ([], []), (np.array([[0], [1], [4]]), [9, 8]),
                    (torch.tensor([0, 1, 4, -7]), torch.tensor([9, 8]))):
        for opts in (F.make_opts(kv_bits=8), None):
            p = F.flex_attn_plan(SHAPE, opts, qsl, ls, 4)
            assert p.batch == ((2, 4) if len(ls) else (0, 0)) and p.info["num_seqs"] == len(ls)


def test_arguments_keep_their_tensors():
    """The calls read them by their addresses: a table made in place, or a view
    that no one else holds, stays until the arguments go."""
    import gc
    import weakref
    t = tensors()
    kc = torch.zeros(4, 16, 4, 128, dtype=torch.bfloat16)
    bad, lse, pos = torch.zeros(1, dtype=torch.int32), torch.zeros(3, 28), torch.zeros(3, dtype=torch.int32)
    append = (t["k_new"], t["v_new"], t["bt"], t["ls"], t["qsl"], t["k"], t["v"], t["s"], t["q"], t["q_out"], bad)
    for make, given in ((F.make_rope, (F.rope_table(64, 128, device="cpu"), pos)),
                        (F.make_rope_append_args, (t["q"], t["q_out"], t["k_new"], t["v_new"], pos, kc, kc, bad)),
                        (F.make_kv8_append_args, append),
                        (F.make_kv8_args, (t["q"], t["k"], t["v"], t["s"], t["bt"], t["ls"], t["qsl"], t["out"], lse, bad, bad))):
        views = [x[:] for x in given]
        refs, a = [weakref.ref(x) for x in views], make(*views)
        del views
        gc.collect()
        assert all(r() is not None for r in refs), make.__name__
        del a
        gc.collect()
        assert not any(r() is not None for r in refs), make.__name__


def test_a_plan_is_copied_on_its_own_device(monkeypatch):
    """The upload goes to the stream of the device that holds the plan's copy,
    which is the one that the run calls take, whatever device is current."""
    import contextlib
    seen = []

    @contextlib.contextmanager
    def on(dev):
        seen.append(("enter", dev))
        yield
        seen.append(("leave", dev))

    monkeypatch.setattr(torch.cuda, "device", on)
    monkeypatch.setattr(F, "flex_attn_plan_upload", lambda plan, d_plan, stream=None: seen.append(("copy", d_plan.device)))
    F.PagedAttention(F.make_shape(28, 4, 128, 128, 16, 0.1), F.make_opts(kv_bits=8), [0, 1], [40], 3, device="cpu")
    dev = torch.device("cpu")
    assert seen == [("enter", dev), ("copy", dev), ("leave", dev)]


class _Stream:
    """A stream of torch's, by its handle; what is done with it is logged."""
    def __init__(self, handle, log, device=None):
        self.cuda_stream, self.log = handle, log

    def record_event(self):
        self.log.append(("record", self.cuda_stream))
        return "the copy's event"

    def wait_event(self, event):
        self.log.append(("wait", self.cuda_stream, event))


def test_a_run_on_another_stream_waits_for_the_plans_copy(monkeypatch):
    """Every run call, once a stream: not on the stream that the copy is queued
    on, and not in a capture."""
    import contextlib
    log, capturing = [], [False]
    monkeypatch.setattr(torch.cuda, "device", lambda d: contextlib.nullcontext())
    monkeypatch.setattr(torch.cuda, "stream", lambda s: contextlib.nullcontext())
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda d=None: _Stream(5, log))
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda h, device=None: _Stream(h, log))
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: capturing[0])
    copy = F._PlanCopy(torch.device("cuda:0"))
    assert log == [("record", 5)]

    class Lib:
        def __getattr__(self, name):
            return lambda *a: log.append(name) or F.FLEX_OK

    monkeypatch.setattr(F, "lib", lambda: Lib())
    t = tensors()
    a = F.make_kv8_args(t["q"], t["k"], t["v"], t["s"], t["bt"], t["ls"], t["qsl"], t["out"])
    a.device, a.plan_copy = torch.device("cuda:0"), copy

    class P:
        handle, shape, batch = None, SHAPE, (2, 3)

    a16 = F.Args()
    a16.plan_copy = copy
    calls = [(F.flex_attn_decode, (P, a16)), (F.flex_attn_prefill, (P, a16)), (F.flex_attn_mixed, (P, a16, 0)),
             (F.flex_attn_mixed_static, (P, a16, 0)), (F.flex_attn_decode_kv8, (P, a)), (F.flex_attn_prefill_kv8, (P, a)),
             (F.flex_attn_mixed_kv8, (P, a, 0))]
    for i, (call, args) in enumerate(calls):
        name, side, null = call.__name__, 100 + i, ctypes.c_void_p(200 + i)
        del log[:]
        call(*args)
        call(*args, stream=5)
        assert log == [name, name], name                       # the copy's own stream
        capturing[0] = True
        call(*args, stream=side)
        capturing[0] = False
        assert log[2:] == [name], name                         # a capture, which must not wait
        call(*args, stream=side)
        call(*args, stream=side)
        call(*args, stream=null)
        assert log[3:] == [("wait", side, "the copy's event"), name, name, ("wait", null.value, "the copy's event"), name], name
    for shape, bits, make in ((SHAPE, 8, "kv8_args"), (SHAPE, 16, "args")):
        monkeypatch.undo()
        with monkeypatch.context() as m:
            m.setattr(torch.cuda, "device", lambda d: contextlib.nullcontext())
            m.setattr(F, "flex_attn_plan_upload", lambda plan, d_plan, stream=None: None)
            pa = F.PagedAttention(shape, F.make_opts(kv_bits=bits), t["qsl"], t["ls"], 3, device="cpu")
        kc = torch.zeros(t["k"].shape, dtype=torch.bfloat16)
        cache = (t["k"], t["v"], t["s"]) if bits == 8 else (kc, kc)
        assert getattr(pa, make)(t["q"], *cache, t["bt"], t["ls"], t["qsl"], t["out"]).plan_copy is pa.plan_copy
