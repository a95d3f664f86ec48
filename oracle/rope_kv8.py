"""CPU oracle for rotary positions on the way into the KV pool, and for its 8-bit form.

TEST INFRASTRUCTURE. Only ``tests/`` imports this module. The library never
does, and this module imports nothing from the library.

What it computes. Co-located prefill and decode extend and read one shared KV
pool in place (Sec. 3.4, "Memory Locality"); the paper gives neither a position
encoding nor a cache type, so these are the plain definitions:

* rotation: pair i of a head's rotated part, values (x, y), becomes
  (x c - y s, y c + x s) with c and s of its position from a table [position]
  [cosines of all pairs, then sines]; pairs lie half a part apart or side by
  side; with several axes a pair goes by one axis's position.
* 8-bit blocks: 16 consecutive slots of a page, one KV head, K or V. A call's
  new rows of a block set the scale 2^k: the least k >= -117 with every finite
  magnitude <= 448 * 2^k, not below the block's scale when its first new row is
  not row 0 (it then holds earlier rows, which are coded again if the scale
  grew). Codes are e4m3 (4 exponent bits, bias 7, 3 fraction bits, no infinity,
  0x7F NaN), rounded to nearest even; what is not finite becomes NaN.

``dtype`` chooses the arithmetic of the rotation: float64, or float32 with each
product and sum rounded (what the 8-bit codes are defined on).

Pins: tests/test_kv8_cpu.py.
"""
from __future__ import annotations

import math

import numpy as np


def axis_of_pairs(pairs, sections, dealt):
    """The axis each pair goes by."""
    if not sections or len(sections) == 1:
        return [0] * pairs
    if not dealt:
        return [a for a, n in enumerate(sections) for _ in range(n)]
    axes, left = [], list(sections)
    for i in range(pairs):
        a = i % len(sections)
        if a and left[a]:
            left[a] -= 1
        else:
            a = 0
        axes.append(a)
    return axes


def rotate(x, table, positions, begin=0, neighbours=False, sections=None, dealt=False, dtype=np.float64):
    """x [tokens, heads, d] turned; positions [axes, tokens]; table [max_position, rot_dim]."""
    x = np.asarray(x, dtype=dtype).copy()
    rot = table.shape[1]
    pairs = rot // 2
    for i, a in enumerate(axis_of_pairs(pairs, sections, dealt)):
        c = np.asarray(table[positions[a], i], dtype=dtype)[:, None]
        s = np.asarray(table[positions[a], pairs + i], dtype=dtype)[:, None]
        u = begin + (2 * i if neighbours else i)
        w = u + (1 if neighbours else pairs)
        xu, xw = x[:, :, u].copy(), x[:, :, w].copy()
        x[:, :, u] = xu * c - xw * s
        x[:, :, w] = xw * c + xu * s
    return x


def decode_table():
    """Value of each of the 256 codes."""
    v = np.empty(256)
    for c in range(256):
        e, f = (c >> 3) & 15, c & 7
        m = math.ldexp(8 + f, e - 10) if e else math.ldexp(f, -9)
        v[c] = math.nan if (c & 127) == 127 else (-m if c >> 7 else m)
    return v


VALUES = decode_table()


def encode(x):
    """Codes of values (finite ones up to 448): to nearest, ties to the even code."""
    x = np.asarray(x, dtype=np.float64)
    mags = VALUES[:127]                                    # ascending, code = index
    a = np.minimum(np.abs(np.where(np.isfinite(x), x, 0.0)), 448.0)
    lo = np.clip(np.searchsorted(mags, a, side="right") - 1, 0, 125)
    down, up = a - mags[lo], mags[lo + 1] - a
    code = np.where((up < down) | ((up == down) & (lo % 2 == 1)), lo + 1, lo)
    code = np.where(np.signbit(x), code | 128, code)
    return np.where(np.isfinite(x), code, 127).astype(np.uint8)


def scale_exponent(largest):
    """Least k >= -117 with largest <= 448 * 2^k."""
    k = -117
    while largest > 448.0 * 2.0 ** k:
        k += 1
    return k


def kv8_append(codes, scales, rows, block_table, seq_lens, qsl, page_size):
    """Append new rows [tokens, Hkv, d] (float32 values) of one of K / V.

    codes [pages, P, Hkv, d] and scales [pages, P / 16, Hkv] (bytes) are not
    modified; returns the new ones. Every token must be in range."""
    codes, scales = codes.copy(), scales.copy()
    for s in range(len(seq_lens)):
        q0, q1, L = int(qsl[s]), int(qsl[s + 1]), int(seq_lens[s])
        start = L - (q1 - q0)
        for b in range(start // 16, -(-L // 16)):
            first, last = max(start, 16 * b), min(L, 16 * b + 16)
            if first >= last:
                continue
            page, slot0 = int(block_table[s][16 * b // page_size]), 16 * b % page_size
            new = np.asarray(rows[q0 + first - start:q0 + last - start], dtype=np.float64)
            for h in range(codes.shape[2]):
                finite = np.abs(new[:, h][np.isfinite(new[:, h])])
                k = scale_exponent(finite.max() if finite.size else 0.0)
                if first > 16 * b:
                    old = int(scales[page, slot0 // 16, h]) - 127
                    held = slice(slot0, slot0 + first - 16 * b)
                    if k > old:
                        codes[page, held, h] = encode(VALUES[codes[page, held, h]] * 2.0 ** (old - k))
                    k = max(k, old)
                codes[page, slot0 + first - 16 * b:slot0 + last - 16 * b, h] = encode(new[:, h] / 2.0 ** k)
                scales[page, slot0 // 16, h] = k + 127
    return codes, scales


def values(codes, scales):
    """Cached values [pages, P, Hkv, d] of codes and scales [pages, P / 16, Hkv]."""
    k = np.repeat(scales.astype(np.int64) - 127, 16, axis=1)[..., None]
    return np.where(np.repeat(scales, 16, axis=1)[..., None] == 255, np.nan, np.ldexp(VALUES[codes], k))
