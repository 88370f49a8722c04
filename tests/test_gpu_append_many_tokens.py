"""snapkv_append_paged on both sides of 1024 tokens, from where on a wave goes through all heads of its token: queries, keys, their
second copy and pages against the oracle's rotation; bounds in serve_checks.py."""
import numpy as np
import pytest
import torch

from oracle import serve_oracle as orc
from serve_checks import DT, W24, half_step, num, offsets, pool, rows, seeded, tables

pytestmark = pytest.mark.gpu


def turned(x, pos, cos, sin, interleaved):
    """The oracle's rotation, a position at a time for all tokens there, and |a| + |b| of each element's pair."""
    out, size, half = np.empty_like(x), np.zeros_like(x), cos.shape[1]
    for p in np.unique(pos):
        at = np.flatnonzero(pos == p)
        # (heads and tokens are alike to a rotation)
        out[at] = orc.rotate(x[at].reshape(1, -1, x.shape[-1]), [p], cos, sin, interleaved).reshape(len(at), *x.shape[1:])
    for m in range(half):
        i, j = (2 * m, 2 * m + 1) if interleaved else (m, m + half)
        size[..., i] = size[..., j] = np.abs(x[..., i]) + np.abs(x[..., j])
    return out, size


def close(got, want, size, dtype):
    bound = half_step(dtype) * np.abs(want) + 4 * W24 * size + (2.0 ** -25 if dtype == torch.float16 else 1e-38)
    err = np.abs(num(got) - want)
    assert (err <= bound).all(), float((err / bound).max())


CASES = [   # lengths, Hq, Hkv, D, dtype, rot, interleaved, layout
    ([1000, 23], 32, 8, 128, "bf16", 128, False, "fused"),          # 1023 tokens: heads over waves
    ([1000, 24], 32, 8, 128, "bf16", 128, False, "fused"),
    ([7, 0, 1018], 32, 8, 128, "f16", 128, True, "tokens"),
    ([1024], 32, 8, 128, "f32", 128, False, "fused"),
    ([513, 700], 21, 7, 64, "f32", 32, True, "heads"),
    ([1100], 9, 3, 64, "bf16", 64, True, "fused"),
    ([600, 1, 999], 5, 5, 128, "f16", 64, False, "heads"),
    ([1040], 40, 20, 64, "f16", 64, False, "tokens"),
]


@pytest.mark.parametrize("n", range(len(CASES)))
def test_append_matches_oracle(snapkv, n):
    lengths, Hq, Hkv, D, dt, rot, interleaved, layout = CASES[n]
    dtype, gen, T, page = DT[dt], seeded(500 + n), sum(lengths), 16
    q, k, v = (rows(gen, T, h, D, dtype, layout) for h in (Hq, Hkv, Hkv))
    starts = [3 * b for b in range(len(lengths))]
    kp, vp, table = pool(gen, [a + m for a, m in zip(starts, lengths)], page, Hkv, D, dtype, fill=7.0)
    P = 97
    cos, sin = tables(P, rot // 2)
    pos = torch.randint(0, P, (T,), generator=gen, device="cuda").to(torch.int32)
    q_out, k_out = rows(gen, T, Hq, D, dtype, layout), rows(gen, T, Hkv, D, dtype, layout)
    cu, st = offsets(lengths), torch.tensor(starts, dtype=torch.int32, device="cuda")
    old_k, old_v = num(kp), num(vp)
    snapkv.snapkv_append_paged(k, v, kp, vp, table, st, cu_seqlens=cu, positions=pos, cos=cos, sin=sin, interleaved=interleaved,
                               q=q, q_out=q_out, k_out=k_out)
    torch.cuda.synchronize()
    at, c, s = pos.cpu().numpy(), num(cos), num(sin)
    want_q, size_q = turned(num(q), at, c, s, interleaved)
    want_k, size_k = turned(num(k), at, c, s, interleaved)
    close(q_out, want_q, size_q, dtype)
    close(k_out, want_k, size_k, dtype)
    pages_k, pages_v = orc.append(old_k, old_v, want_k, num(v), table.cpu().numpy(), starts, cu.tolist())
    pages_size, _ = orc.append(0 * old_k, 0 * old_v, size_k, num(v), table.cpu().numpy(), starts, cu.tolist())
    close(kp, pages_k, pages_size, dtype)
    assert np.array_equal(num(vp), pages_v)
