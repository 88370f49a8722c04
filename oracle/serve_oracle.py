"""fp64 CPU oracle for the steps around a paged prompt cache: appending tokens, attention over packed prompts, one new token.

TEST INFRASTRUCTURE ONLY.  Nothing in the product imports this file and it imports nothing from the product.

    append    logical row r = starts[b] + i of sequence b's i-th new token lies in row r % page of page table[b][r / page];
              keys and queries are turned by their position p: each pair (x_i, x_j), (i, j) = (m, m + R/2) or (2m, 2m + 1),
              becomes (x_i cos - x_j sin, x_j cos + x_i sin) with row p of the tables, for m < R/2
    prompt    out[i, h] = sum_{j <= i} softmax_j(q[i, h] . k[j, h // g] / sqrt(D)) v[j, h // g], lse[h, i] the logarithm of
              the sum of exponentials, within each of the packed prompts
    decode    the same for one query per sequence over the first lens[b] rows that the block table names

All in float64 on the exact stored values.  The attentions also return what bounds rounding errors: the mean of |v| under the
same probabilities and the largest sum of |q_d k_d| / sqrt(D) behind a logit.

Pins (tests/test_serve_oracle_pins.py): position 0, a quarter turn and the sum of two turns written by hand, dot products
that depend on position differences only, interleaved pairs against a permutation of the others, zero queries (running
means), one token, scipy's softmax and logsumexp, the last row of a prompt against the step over pages, and pages
against plain indexing.  No function is unpinned.
"""
from __future__ import annotations

import numpy as np


def rotate(x, positions, cos, sin, interleaved):
    """x [T, H, D], positions [T], cos and sin [P, R/2] -> the turned rows."""
    x = np.array(x, dtype=np.float64)
    half = cos.shape[1]
    for t, p in enumerate(positions):
        p = min(max(int(p), 0), cos.shape[0] - 1)
        for m in range(half):
            i, j = (2 * m, 2 * m + 1) if interleaved else (m, m + half)
            a, b = x[t, :, i].copy(), x[t, :, j].copy()
            x[t, :, i] = a * cos[p, m] - b * sin[p, m]
            x[t, :, j] = b * cos[p, m] + a * sin[p, m]
    return x


def append(k_pages, v_pages, k, v, table, starts, cu):
    """The pages after the tokens' rows (rotated already) went in; tokens of no sequence and rows without a page are skipped."""
    k_pages, v_pages = np.array(k_pages, dtype=np.float64), np.array(v_pages, dtype=np.float64)
    pages, page = k_pages.shape[:2]
    for b in range(len(starts)):
        for t in range(int(cu[b]), int(cu[b + 1])):
            r = int(starts[b]) + t - int(cu[b])
            if r < 0 or r // page >= table.shape[1] or not 0 <= table[b, r // page] < pages:
                continue
            k_pages[table[b, r // page], r % page] = k[t]
            v_pages[table[b, r // page], r % page] = v[t]
    return k_pages, v_pages


def _attend(q, k, v):
    """One query over all rows: out [D], lse, the mean of |v|, the largest sum of |q k| / sqrt(D)."""
    s = k @ q / np.sqrt(float(q.size))
    m = s.max()
    e = np.exp(s - m)
    z = e.sum()
    return e @ v / z, m + np.log(z), e @ np.abs(v) / z, (np.abs(k) @ np.abs(q)).max() / np.sqrt(float(q.size))


def prompt_attention(q, k, v, cu):
    """q [T, Hq, D], k and v [T, Hkv, D], cu [B + 1] -> out, lse [Hq, T], mean |v|, reach [Hq, T]; rows of no prompt are NaN."""
    q, k, v = (np.asarray(x, dtype=np.float64) for x in (q, k, v))
    T, Hq, D = q.shape
    g = Hq // k.shape[1]
    out, spread = np.full(q.shape, np.nan), np.full(q.shape, np.nan)
    lse, reach = np.full((Hq, T), np.nan), np.full((Hq, T), np.nan)
    for a, e in zip(cu[:-1], cu[1:]):
        n = int(e) - int(a)
        if n <= 0:
            continue
        seen = np.tril(np.ones((n, n), dtype=bool))
        for h in range(Hq):
            qh, kh, vh = q[a:e, h], k[a:e, h // g], v[a:e, h // g]
            s = np.where(seen, qh @ kh.T / np.sqrt(float(D)), -np.inf)
            m = s.max(axis=1, keepdims=True)
            p = np.exp(s - m)
            z = p.sum(axis=1, keepdims=True)
            out[a:e, h] = p @ vh / z
            lse[h, a:e] = (m + np.log(z))[:, 0]
            spread[a:e, h] = p @ np.abs(vh) / z
            reach[h, a:e] = np.where(seen, np.abs(qh) @ np.abs(kh).T, 0.0).max(axis=1) / np.sqrt(float(D))
    return out, lse, spread, reach


def decode_paged(q, k_pages, v_pages, table, lens):
    """q [B, Hq, D], pages [P, page, Hkv, D], table [B, columns], lens [B] -> out, lse [B, Hq], mean |v|, reach [B, Hq]."""
    q = np.asarray(q, dtype=np.float64)
    B, Hq, D = q.shape
    pages, page, Hkv, _ = k_pages.shape
    out, spread = np.zeros(q.shape), np.zeros(q.shape)
    lse, reach = np.full((B, Hq), -np.inf), np.zeros((B, Hq))
    for b in range(B):
        S = int(lens[b])
        if S <= 0:
            continue
        at = np.clip(table[b, np.arange(S) // page], 0, pages - 1)
        for h in range(Hq):
            kh = np.asarray(k_pages[at, np.arange(S) % page, h * Hkv // Hq], dtype=np.float64)
            vh = np.asarray(v_pages[at, np.arange(S) % page, h * Hkv // Hq], dtype=np.float64)
            out[b, h], lse[b, h], spread[b, h], reach[b, h] = _attend(q[b, h], kh, vh)
    return out, lse, spread, reach
