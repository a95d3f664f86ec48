"""Batches and tensors for the tests of rotary positions and of the 8-bit cache."""
import math

import numpy as np
import torch

import oracle.rope_kv8 as RK
from paper_2606_04415_amd import flexattn as F


def batch(ns, ls, P, seed, spare=3, width=0):
    """Block table over a pool in random order (entries past a sequence: a
    page of no sequence), seq_lens, query_start_loc, pages of the pool."""
    r = np.random.RandomState(seed)
    per = [-(-L // P) for L in ls]
    pages = sum(per) + spare
    order = r.permutation(pages)
    bt = np.full((len(ls), max(per + [1]) + width), order[-1], dtype=np.int32)
    at = 0
    for s, n in enumerate(per):
        bt[s, :n] = order[at:at + n]
        at += n
    qsl = np.concatenate([[0], np.cumsum(ns)]).astype(np.int32)
    return bt, np.array(ls, dtype=np.int32), qsl, pages


def bf16(shape, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(torch.bfloat16)


def table(max_position, rot_dim):
    return F.rope_table(max_position, rot_dim, 1e4, device="cpu")


def cache8(pages, P, hkv, d, seed, spread=3):
    """Codes that fill the type's range and scales that differ by 2^spread, on the host (bytes)."""
    r = np.random.RandomState(seed)
    k, v = (RK.encode(r.randn(pages, P, hkv, d) * 112) for _ in "kv")
    return k, v, r.randint(119, 119 + spread, size=(pages, P // 16, hkv, 2)).astype(np.uint8)


def poison(k, v, scales, bt, ls, P):
    """NaN codes in every slot that no sequence uses, and NaN scales in every block that none does."""
    used = np.zeros(k.shape[:2], dtype=bool)
    for s, L in enumerate(ls):
        for t in range(L):
            used[bt[s, t // P], t % P] = True
    k[~used], v[~used] = 127, 255
    scales[~used.reshape(used.shape[0], -1, 16).any(-1)] = 255


def to_gpu(k, v, scales):
    return (torch.from_numpy(k).cuda().view(torch.float8_e4m3fn), torch.from_numpy(v).cuda().view(torch.float8_e4m3fn),
            torch.from_numpy(scales).cuda().view(torch.float8_e8m0fnu))


def attend64(q, k, v, bt, ls, qsl, sm_scale):
    """Attention in 64 bits from its definition, one sequence at a time: out,
    lse, the same sum over |v| (what the roundings of the probabilities are
    weighed by) and the largest sum |q| |k| sm_scale of a row (what the
    roundings of the scores are)."""
    q = q.double().numpy()
    P, hkv = k.shape[1:3]
    G = q.shape[1] // hkv
    out, mag = np.full((2,) + q.shape[:2] + (v.shape[3],), np.nan)
    lse, size = np.full((2,) + q.shape[:2], np.nan)
    for s, L in enumerate(ls):
        n = qsl[s + 1] - qsl[s]
        if n == 0:
            continue
        at = [(bt[s, t // P], t % P) for t in range(L)]
        pg, sl = (np.array(x) for x in zip(*at))
        for h in range(q.shape[1]):
            kk, vv = k[pg, sl, h // G], v[pg, sl, h // G]
            qq = q[qsl[s]:qsl[s + 1], h]
            seen = np.arange(L)[None] <= L - n + np.arange(n)[:, None]
            z = np.where(seen, qq @ kk.T * sm_scale, -np.inf)
            m = z.max(1, keepdims=True)
            e = np.exp(z - m)
            l = e.sum(1, keepdims=True)
            rows = slice(qsl[s], qsl[s + 1])
            out[rows, h], mag[rows, h] = e @ vv / l, e @ np.abs(vv) / l
            lse[rows, h] = (m + np.log(l))[:, 0]
            size[rows, h] = (np.where(seen, np.abs(qq) @ np.abs(kk).T, 0) * sm_scale).max(1)
    return out, lse, mag, size


def check_attention(out, lse, ref, ls, qsl, d, what):
    """Bounds from the arithmetic. Scores: products of bf16 values are exact in
    fp32 and d + 8 sums and scalings round, each by 2^-24 of at most `size`:
    dz = (d + 8) 2^-24 size. Row sums: at most L + 64 additions and one
    exponential (2 ulp) each. So probabilities are off by dp = dz + 2^-22 and
    sums by ds = dp + (L + 64) 2^-24, relatively. Outputs: a probability is
    rounded once more to bf16 (2^-8) before its product, the sums over L as the
    row sums, and the output is rounded to bf16."""
    ro, rl, mag, size = ref
    L = np.repeat(np.array(ls), np.diff(qsl))[:, None]
    dp = (d + 8) * 2.0 ** -24 * size + 2.0 ** -22
    ds = dp + (L + 64) * 2.0 ** -24
    g = out.double().numpy()
    rows = ~np.isnan(rl[:, 0])
    assert np.isfinite(g[rows]).all(), f"{what}: not finite"
    bound = (2.0 ** -8 + 2 * ds)[..., None] * mag + 2.0 ** -8 * np.abs(ro) + 1e-30
    err = np.abs(g - ro)
    worst = (err / bound)[rows].max() if rows.any() else 0.0
    print(f"  {what}: error at most {worst:.3f} of its bound", flush=True)
    assert worst <= 1.0, f"{what}: {worst:.3f} of the bound"
    if lse is not None:
        e = np.abs(lse.double().numpy() - rl)
        bound = dp + ds + 2.0 ** -22 * np.abs(rl)
        worst = (e / bound)[rows].max() if rows.any() else 0.0
        print(f"  {what}: lse error at most {worst:.3f} of its bound", flush=True)
        assert worst <= 1.0, f"{what}: lse {worst:.3f} of the bound"


def scale_of(d):
    return 1.0 / math.sqrt(d)
