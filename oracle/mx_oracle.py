"""fp64 CPU oracle for microscaled paged caches and for steps whose sequences share prefixes.

TEST INFRASTRUCTURE ONLY.  Nothing in the product imports this file and it imports nothing from the product.

    quantise  a row's values in blocks of 32: e the smallest integer with max |x| <= M 2^e, at least -117 (M = 448 for "fp8", the e4m3
              values, 6 for "fp4", the e2m1 values); scale byte e + 127 and per value the code of the nearest value of the
              element type to x / 2^e, ties to the even code; infinities and NaN: byte 255 and codes 0
    values    what codes and scale bytes stand for: value of the code times 2^(byte - 127), NaN for byte 255
    shared    one query per sequence over its group's prefix rows and then its own

Pins (tests/test_mx_oracle_pins.py): the element values against torch's float8_e4m3fn and a written table, rounding against
that type's conversion, blocks by hand (ties, borders of e, zeros, the smallest e, infinities), values of quantise within half a
step, shared against the step over one table that names both parts.  No function is unpinned.
"""
from __future__ import annotations

import numpy as np

from .serve_oracle import _attend

GRID = {"fp4": np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]),
        "fp8": np.array([(m / 8.0 if e == 0 else 1 + m / 8.0) * 2.0 ** (max(e, 1) - 7) for e in range(16) for m in range(8)][:-1])}


def quantise(x, kind):
    """x [..., D] -> codes [..., D] (one per value, sign in the bit above the magnitude's) and scale bytes [..., D / 32], as integers."""
    grid = GRID[kind]
    sign_bit = 128 if kind == "fp8" else 8
    x = np.asarray(x, dtype=np.float64)
    blocks = x.reshape(x.shape[:-1] + (-1, 32))
    large = np.abs(blocks).max(axis=-1)
    lost = ~np.isfinite(large)                              # (NaN is the largest of any block)
    safe = np.where(lost | (large == 0), 1.0, large)
    e = np.floor(np.log2(safe / grid[-1])).astype(np.int64) - 1
    for _ in range(3):
        e = e + (safe > np.ldexp(grid[-1], e))
    e = np.where(large == 0, -117, np.maximum(e, -117))
    y = np.ldexp(np.where(lost[..., None], 0.0, blocks), -e[..., None])
    mag = np.abs(y)
    hi = np.clip(np.searchsorted(grid, mag), 1, len(grid) - 1)
    up, down = grid[hi] - mag, mag - grid[hi - 1]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, hi - 1)
    code = code + sign_bit * np.signbit(y)
    return code.reshape(x.shape), np.where(lost, 255, e + 127)


def values(codes, scales, kind):
    """codes [..., D], one per value, and scale bytes [..., D / 32] -> float64."""
    sign_bit = 128 if kind == "fp8" else 8
    grid = np.append(GRID[kind], np.nan) if kind == "fp8" else GRID[kind]
    codes, scales = np.asarray(codes, dtype=np.int64), np.asarray(scales, dtype=np.int64)
    x = grid[codes % sign_bit] * np.where(codes >= sign_bit, -1.0, 1.0)
    unit = np.where(scales == 255, np.nan, np.ldexp(1.0, np.minimum(scales, 254) - 127))
    return x * np.repeat(unit, 32, axis=-1)


def pack(codes, kind):
    """One code per value -> bytes as they lie in pages."""
    codes = np.asarray(codes, dtype=np.uint8)
    return codes if kind == "fp8" else codes[..., 0::2] | (codes[..., 1::2] << 4)


def unpack(raw, kind):
    raw = np.asarray(raw, dtype=np.uint8)
    return raw if kind == "fp8" else np.stack([raw & 15, raw >> 4], axis=-1).reshape(raw.shape[:-1] + (-1,))


def decode_shared(q, k_pages, v_pages, prefix_table, prefix_lens, table, lens, groups):
    """q [B, Hq, D], pages [P, page, Hkv, D], groups: (first, last) sequences of each -> out, lse [B, Hq], mean |v|, reach [B, Hq]."""
    q = np.asarray(q, dtype=np.float64)
    B, Hq, D = q.shape
    pages, page, Hkv, _ = k_pages.shape
    out, spread = np.zeros(q.shape), np.zeros(q.shape)
    lse, reach = np.full((B, Hq), -np.inf), np.zeros((B, Hq))

    def named(row, n):
        j = np.arange(max(0, int(n)))
        return np.clip(row[j // page], 0, pages - 1), j % page

    for b in range(B):
        parts = [named(prefix_table[i], prefix_lens[i]) for i, (a, e) in enumerate(groups) if a <= b < e] + [named(table[b], lens[b])]
        at, line = (np.concatenate(x) for x in zip(*parts))
        if len(at) == 0:
            continue
        for h in range(Hq):
            k, v = (np.asarray(t[at, line, h * Hkv // Hq], dtype=np.float64) for t in (k_pages, v_pages))
            out[b, h], lse[b, h], spread[b, h], reach[b, h] = _attend(q[b, h], k, v)
    return out, lse, spread, reach
