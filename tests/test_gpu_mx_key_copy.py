"""The keys' second copy of snapkv_append_paged_mx: the rotation in 64 bits, rounded once to the call's type.

Products of 24 bits at most are exact in 64, and their sum is off by 2^-53 of itself.  So the copy lies between both ends of that interval, rounded: they are
one number but where a middle between two lies within it.
"""
import math

import numpy as np
import pytest
import torch

from serve_checks import DT, offsets, rows, seeded, tables
from test_gpu_mx_cache import empty_pool

pytestmark = pytest.mark.gpu


def turned(x, cos, sin, inter):
    """Both ends of the interval that the rotation of x [T, H, D] lies in, in numpy's longest type; cos, sin [T, D / 2]."""
    x, c, s = (np.asarray(a, dtype=np.longdouble) for a in (x, cos[:, None], sin[:, None]))
    D = x.shape[-1]
    a, b = (x[..., 0::2], x[..., 1::2]) if inter else (x[..., :D // 2], x[..., D // 2:])
    lo, hi = np.empty_like(x), np.empty_like(x)
    for i, (p, q) in enumerate(((a * c, -b * s), (b * c, a * s))):
        off = np.ldexp(np.abs(p) + np.abs(q), -52)
        at = (..., slice(i, None, 2)) if inter else (..., slice(i * D // 2, (i + 1) * D // 2))
        lo[at], hi[at] = p + q - off, p + q + off
    return lo, hi


def nearest(x, dtype):
    """x rounded to nearest even, once (torch's conversion of float64 goes by way of float32); no number here is as large as the type's largest."""
    bits = {torch.float32: 24, torch.bfloat16: 8, torch.float16: 11}[dtype]
    least = math.log2(torch.finfo(dtype).smallest_normal)
    step = np.maximum(np.frexp(x)[1], int(least) + 1) - bits
    return torch.from_numpy(np.ldexp(np.rint(np.ldexp(x, -step)), step).astype(np.float64))


@pytest.mark.parametrize("T", [5, 1100])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
def test_copy_is_rounded_once(snapkv, dt, inter, T):
    gen, H, D, dtype = seeded(T), 2, 128, DT[dt]
    k, v = (rows(gen, T, H, D, dtype, "tokens") for _ in range(2))
    pool = empty_pool(-(-T // 16), 16, H, D, "fp8")
    table = torch.arange(len(pool[0]), dtype=torch.int32, device="cuda").view(1, -1)
    cos, sin = tables(T, D // 2)
    k_out = torch.empty_like(k)
    snapkv.snapkv_append_paged_mx(k, v, *pool, table, torch.zeros(1, dtype=torch.int32, device="cuda"), cu_seqlens=offsets([T]), cos=cos, sin=sin,
                                  interleaved=inter, k_out=k_out)
    torch.cuda.synchronize()
    lo, hi = turned(k.double().cpu().numpy(), cos.double().cpu().numpy(), sin.double().cpu().numpy(), inter)
    lo, hi = (nearest(x, dtype) for x in (lo, hi))                                         # (roundings keep the order)
    got = k_out.double().cpu()
    assert ((lo <= got) & (got <= hi)).all() and float((lo != hi).float().mean()) < 1e-4


def test_copy_beyond_the_range_is_infinite(snapkv):
    """As a float32 sum is; the codes are those of the largest number."""
    D = 64
    k = torch.full((1, 1, D), 3.0e38, device="cuda")
    cos, sin = (torch.full((1, D // 2), x, device="cuda") for x in (0.8, 0.6))
    pool = empty_pool(1, 16, 1, D, "fp8")
    zero, k_out = torch.zeros((1, 1), dtype=torch.int32, device="cuda"), torch.empty_like(k)
    snapkv.snapkv_append_paged_mx(k, k, *pool, zero, zero[0], cos=cos, sin=sin, k_out=k_out)
    ko, vo = torch.empty_like(k), torch.empty_like(k)
    snapkv.snapkv_read_paged_mx(*pool, zero, zero[0], ko, vo)
    torch.cuda.synchronize()
    assert (k_out[..., D // 2:] == float("inf")).all() and k_out[..., :D // 2].isfinite().all()
    assert int(pool[1][0, 0, 0, 1]) == 127 + 120             # (448 2^120 is the first above 2^128 (1 - 2^-24))
