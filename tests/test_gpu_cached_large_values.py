"""Steps over cached rows whose values are near float32's and bfloat16's largest: means of finite numbers are finite, and the oracle's.

Bounds in mx_checks.py; a key's logit is 16 k[0] / sqrt(D) plus the products of small numbers, so rows climb as the test says.
"""
import math

import numpy as np
import pytest
import torch

from mx_checks import check_step, mx_values
from oracle import mx_oracle as orc
from serve_checks import num, offsets, seeded

pytestmark = pytest.mark.gpu

LARGEST = torch.finfo(torch.bfloat16).max


def pages_of(gen, rows, Hkv, D, kind, climb, every):
    """Pages of 16 rows, in order; every `every`-th key from row 128 on has a logit 2^climb above the others', values are of 2^120 to 2^124."""
    k = 0.01 * torch.randn((rows, Hkv, D), generator=gen, device="cuda")
    top = (torch.arange(rows, device="cuda") >= 128) & (torch.arange(rows, device="cuda") % every == 0)
    k[..., 0] = torch.where(top, climb * math.log(2) * math.sqrt(D) / 16, 0.0)[:, None]
    v = 2.0 ** 122 * torch.randn((rows, Hkv, D), generator=gen, device="cuda").clamp(-3.5, 3.5)
    if kind == "plain":
        return [x.to(torch.bfloat16).view(-1, 16, Hkv, D) for x in (k, v)], [x.to(torch.bfloat16).double().cpu().numpy().reshape(-1, 16, Hkv, D) for x in (k, v)]
    parts, values = [], []
    for x in (k, v):
        codes, scales = orc.quantise(num(x), kind)
        parts += [torch.from_numpy(a.astype(np.uint8)).cuda().view(-1, 16, Hkv, a.shape[-1]) for a in (orc.pack(codes, kind), scales)]
        values.append(mx_values(*parts[-2:], kind))
    return parts, values


def queries(gen, B, Hq, D):
    q = 0.5 * torch.randn((B, Hq, D), generator=gen, device="cuda")
    q[..., 0] = 16
    return q.to(torch.bfloat16)


@pytest.mark.parametrize("climb", [7, 9.5, 18])
@pytest.mark.parametrize("members", [1, 6, 12, 30])
@pytest.mark.parametrize("kind", ["plain", "fp8", "fp4"])
def test_shared_prefix_of_large_values(snapkv, kind, members, climb):
    """Tiles of 16, 32, 64 and 128 query heads, own rows that climb too."""
    gen, Hq, Hkv, D, P, own = seeded(int(10 * climb) + members), 8, 2, 128, 512, 256
    pages, (k, v) = pages_of(gen, P + own, Hkv, D, kind, climb, 40)
    kw = dict(zip(("k_pages", "v_pages") if kind == "plain" else ("k_pages", "k_scales", "v_pages", "v_scales"), pages))
    q = queries(gen, members, Hq, D)
    prefix_table = torch.arange(P // 16, dtype=torch.int32, device="cuda").view(1, -1)
    table = torch.arange(P // 16, (P + own) // 16, dtype=torch.int32, device="cuda").repeat(members, 1)
    prefix_lens = torch.tensor([P], dtype=torch.int32, device="cuda")
    lens = torch.tensor([own - 3 * i for i in range(members)], dtype=torch.int32, device="cuda")
    out, lse = torch.empty_like(q), torch.empty((members, Hq), device="cuda")
    snapkv.snapkv_decode_attention_shared(q=q, prefix_table=prefix_table, prefix_lens=prefix_lens, max_prefix=P, block_table=table, lens=lens, max_len=own,
                                          out=out, out_lse=lse, cu_groups=offsets([members]), **kw)
    torch.cuda.synchronize()
    want = orc.decode_shared(num(q), k, v, prefix_table.cpu().numpy(), [P], table.cpu().numpy(), lens.tolist(), [(0, members)])
    check_step(out, lse, *want, P + own, q.dtype, plain=kind == "plain", rounded=members * Hq // Hkv > 32)


@pytest.mark.parametrize("climb", [7, 9.5])
@pytest.mark.parametrize("n", [300, 2100])
@pytest.mark.parametrize("kind", ["fp8", "fp4"])
def test_step_over_large_values(snapkv, kind, n, climb):
    gen, Hq, Hkv, D, B = seeded(n), 8, 2, 128, 3
    rows = -(-n // 16) * 16
    (kc, ks, vc, vs), (k, v) = pages_of(gen, rows, Hkv, D, kind, climb, 40)
    q = queries(gen, B, Hq, D)
    table = torch.arange(rows // 16, dtype=torch.int32, device="cuda").repeat(B, 1)
    lens = torch.tensor([n, n - 1, n - 77], dtype=torch.int32, device="cuda")
    out, lse = torch.empty_like(q), torch.empty((B, Hq), device="cuda")
    snapkv.snapkv_decode_attention_paged_mx(q, kc, ks, vc, vs, table, lens, n, out, lse)
    torch.cuda.synchronize()
    want = orc.decode_shared(num(q), k, v, np.zeros((1, 1), np.int32), [0], table.cpu().numpy(), lens.tolist(), [])
    check_step(out, lse, *want, n, q.dtype)


@pytest.mark.parametrize("members", [1, 6, 12, 30])
def test_mean_of_the_largest_values_is_finite(snapkv, members):
    """Every 32nd key's probability is a power of two, the others' lie just above a middle between two bfloat16 numbers: rounded they sum up to 2^-8
    more than they are, and a mean of the largest number would be an infinity."""
    gen, Hq, Hkv, D, P = seeded(members), 8, 2, 128, 512
    k = torch.zeros((P, Hkv, D), device="cuda")
    x = math.log2(0.5 * (1 + 2.0 ** -8 + 2.0 ** -10)) * math.log(2) * math.sqrt(D)    # q . k
    rough = float(torch.tensor(x).to(torch.bfloat16))
    others = torch.arange(P, device="cuda") % 32 != 0
    k[others, :, 0], k[others, :, 1] = rough, (x - rough) * 64
    q = torch.zeros((members, Hq, D), device="cuda")
    q[..., 0], q[..., 1] = 1, 1 / 64
    q = q.to(torch.bfloat16)
    k = k.to(torch.bfloat16).view(-1, 16, Hkv, D)
    v = torch.full_like(k, LARGEST)
    out = torch.empty_like(q)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    snapkv.snapkv_decode_attention_shared(q=q, k_pages=k, v_pages=v, prefix_table=torch.arange(P // 16, dtype=torch.int32, device="cuda").view(1, -1),
                                          prefix_lens=i32(P), max_prefix=P, block_table=torch.zeros((members, 1), dtype=torch.int32, device="cuda"),
                                          lens=i32(*[0] * members), max_len=1, out=out, cu_groups=offsets([members]))
    torch.cuda.synchronize()
    assert out.isfinite().all() and (out.double() >= LARGEST * (1 - 2.0 ** -7)).all()


@pytest.mark.parametrize("climb", [0, 7, 9.5])
@pytest.mark.parametrize("members", [1, 6, 12, 30])
def test_small_values_keep_their_bits(snapkv, members, climb):
    """Values of 2^-112 to 2^-111: a probability is at least 2^-16 where it counts, their products are at least 2^-128 and lose 2^-150 each, 2^-22 of
    themselves, so the answer is off by its rounding, 2^-8, and that of the probabilities, 2^-8 at most."""
    gen, Hq, Hkv, D, P = seeded(members), 8, 2, 128, 512
    (k, v), _ = pages_of(gen, P, Hkv, D, "plain", climb, 40)
    v = (2.0 ** -112 * (1 + torch.rand((P, Hkv, D), generator=gen, device="cuda"))).to(torch.bfloat16).view_as(k)
    q = queries(gen, members, Hq, D)
    out = torch.empty_like(q)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    table = torch.arange(P // 16, dtype=torch.int32, device="cuda").view(1, -1)
    snapkv.snapkv_decode_attention_shared(q=q, k_pages=k, v_pages=v, prefix_table=table, prefix_lens=i32(P), max_prefix=P,
                                          block_table=torch.zeros((members, 1), dtype=torch.int32, device="cuda"), lens=i32(*[0] * members), max_len=1,
                                          out=out, cu_groups=offsets([members]))
    torch.cuda.synchronize()
    want, *_ = orc.decode_shared(num(q), num(k), num(v), table.cpu().numpy(), [P], np.zeros((members, 1), np.int32), [0] * members, [(0, members)])
    assert (np.abs(num(out) - want) <= 2.0 ** -7 * want).all()
