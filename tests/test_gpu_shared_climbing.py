"""snapkv_decode_attention_shared in tiles of 64 and 128 query heads where logits climb inside a share: a row's maximum is moved once its sums are not
empty, in some rows of a tile and not in others.  Against the fp64 oracle; bounds in mx_checks.py.

Shares begin at multiples of 128 keys and hold 128 or more; blocks of 32 keys are met in order, all of them by one wave or every other one.  So keys from
64 on of every 128 are the ones that climb, and what the test is about (a climb past the bound up to which a maximum stays, 2^10 or, plain fp16 rows, 2^8,
after a wave's first block) is checked on the host first.
"""
import math

import numpy as np
import pytest
import torch

from mx_checks import mx_values
from oracle import mx_oracle as orc
from serve_checks import DT, num, seeded
from test_gpu_shared_prefix import build, check, run

pytestmark = pytest.mark.gpu

P, LEVEL = 640, 8.0


def climbing(n, members, kind, dtype, D, bits, half):
    """Query heads in turn climb with the keys, hardly notice, and fall; `half`: which keys of eight climb (0: the first four, 1: the others, 2: all)."""
    gen, page = seeded(n), 16
    s = build(gen, [P], [members], [3] * members, page, 8, 2, D, dtype, kind)
    rows = torch.arange(members * 8, device="cuda").view(members, 8)
    s["q"][..., 0] = torch.tensor([LEVEL, 0.5, -LEVEL], device="cuda")[rows % 3].to(dtype)
    j = torch.arange(P, device="cuda")
    k = 0.2 * torch.randn((P, 2, D), generator=gen, device="cuda")
    up = (j % 128 >= 64) & ((half == 2) | (j % 8 // 4 == half))
    k[..., 0] = torch.where(up, bits * math.log(2) * math.sqrt(D) / LEVEL, 0.0)[:, None]
    at = (s["prefix_table"][0, j // page].long(), j % page)
    if kind == "plain":
        s["k_pages"][at] = k.to(dtype)
        seen = num(s["k_pages"][at])
    else:
        codes, scales = orc.quantise(num(k), kind)
        s["k_pages"][at] = torch.from_numpy(orc.pack(codes, kind)).cuda()
        s["k_scales"][at] = torch.from_numpy(scales.astype(np.uint8)).cuda()
        seen = mx_values(s["k_pages"][at], s["k_scales"][at], kind)
    q = num(s["q"])
    logits = np.stack([q[:, h] @ seen[:, h // 4].T for h in range(8)], axis=1) / math.sqrt(D) / math.log(2)
    first = logits.reshape(members, 8, P // 128, 4, 32).max(axis=-1)
    growth = first[..., 2:] - first[..., :2]
    bound = 8 if kind == "plain" and dtype == torch.float16 else 10
    grows = (rows % 3 == 0).cpu().numpy()
    assert (growth[grows] > bound).all() and (growth[~grows] < 6).all()
    return s


@pytest.mark.parametrize("half", [0, 1, 2])
@pytest.mark.parametrize("bits", [12, 27])
@pytest.mark.parametrize("members", [12, 30])
@pytest.mark.parametrize("dt,kind,D", [("bf16", "plain", 128), ("bf16", "plain", 64), ("f16", "plain", 128), ("f16", "plain", 64), ("f16", "fp8", 128),
                                       ("f16", "fp4", 64), ("bf16", "fp4", 128), ("bf16", "fp8", 64)])
def test_rows_that_climb(snapkv, dt, kind, D, members, bits, half):
    s = climbing(7 * members + half, members, kind, DT[dt], D, bits, half)
    check(s, kind, *run(snapkv, s))
