"""What the tests of microscaled pages and shared prefixes share.

Codes and scale bytes are compared exactly: the kernels rotate in 64 bits, where an output is off by at most 2^-52 (|a| + |b|), and round
once.  The oracle rotates in numpy's float64 with the same error, so a code can differ only where a value lies within that of a border
between two codes, which no random input here does, or on a border exactly, where both are exact (position 0).

Attention, with the names of serve_checks.py: keys and values are exact bfloat16 numbers in the products and fp16 queries two bfloat16 parts
whose sum is exact, so logits sum up to 2 D products:  d = 2 (2 D + 4) w reach + 2^-20;  probabilities are two bfloat16 parts by
truncation, c = 2^-14, except for plain fp16 pages, c = 2^-20 (fp16 parts of 2^15 p; what is below 2^-29 of the largest loses up to 2^-39 of
that: n 2^-39 more);  joining m partial sums adds m roundings, m <= n:  |got - want| <= u |want| + (c + 2 d + 3 n w) spread.  Prefixes that more than 32 query heads
of a group meet have their probabilities rounded once, as in the attention over prompts: c = u there (fp16 ones are taken 2^7 times as large, those
that are subnormal then lose up to 2^-32 of the largest each: n 2^-32 more), but for fp16 queries over codes.
"""
import numpy as np
import torch

from oracle import mx_oracle as orc
from serve_checks import W24, half_step, num, pool


def check_step(got, got_lse, want, want_lse, spread, reach, n, dtype, plain=False, rounded=False):
    """got [B, Hq, D], got_lse [B, Hq] tensors (or None), rows that see nothing have want_lse = -inf; n: rows seen at most."""
    some = np.isfinite(want_lse[:, 0])
    got = num(got)
    assert np.isfinite(got).all()
    assert (got[~some] == 0).all()
    D = want.shape[-1]
    c = 2.0 ** -20 + n * 2.0 ** -39 if plain and dtype == torch.float16 else 2.0 ** -14
    if rounded and (plain or dtype == torch.bfloat16):
        c = half_step(dtype) + n * 2.0 ** -32
    d = 2 * (2 * D + 4) * W24 * reach + 2.0 ** -20
    bound = half_step(dtype) * np.abs(want) + (c + 2 * d[..., None] + 3 * n * W24) * spread + 1e-30
    if dtype == torch.float16:
        bound = bound + 2.0 ** -25                               # (half a step of fp16's smallest numbers)
    err = np.abs(got - want)
    assert (err <= bound).all(), (float((err / bound).max()), np.unravel_index((err / bound).argmax(), err.shape))
    if got_lse is not None:
        got_lse = num(got_lse)
        assert np.isneginf(got_lse[~some]).all()
        off = np.abs(got_lse[some] - want_lse[some])
        lse_bound = d[some] + 2 * n * W24 + 2 * W24 * np.abs(want_lse[some])
        assert (off <= lse_bound).all(), float((off / lse_bound).max())


def mx_pool(gen, lens, page, Hkv, D, kind, spare=3):
    """Pages of random codes and scales (bytes of 2^-6 to 2^3) behind a table in random order; unowned rows read as NaN."""
    width = D if kind == "fp8" else D // 2
    _, _, table = pool(gen, lens, page, 1, 1, torch.float32, spare)
    pages = sum(-(-max(0, n) // page) for n in lens) + spare
    out = []
    for _ in range(2):
        codes = torch.full((pages, page, Hkv, width), 0, device="cuda", dtype=torch.uint8)
        scales = torch.full((pages, page, Hkv, D // 32), 255, device="cuda", dtype=torch.uint8)
        for b, n in enumerate(lens):
            j = torch.arange(max(0, n), device="cuda")
            at, line = table[b, j // page].long(), j % page
            c = torch.randint(0, 256, (max(0, n), Hkv, width), generator=gen, device="cuda", dtype=torch.uint8)
            if kind == "fp8":                                    # largest magnitude 15, no NaN
                c = torch.where(c % 128 > 0x57, c & 0x9F, c)
            codes[at, line] = c
            scales[at, line] = torch.randint(121, 126, (max(0, n), Hkv, D // 32), generator=gen, device="cuda", dtype=torch.uint8)
        out += [codes, scales]
    return out, table


def mx_values(codes, scales, kind):
    """Pages as float64 values; what reads as NaN (rows of nobody) as zeros."""
    return np.nan_to_num(orc.values(orc.unpack(codes.cpu().numpy(), kind), scales.cpu().numpy(), kind))
