"""The step over pages where sequences may be far longer than they are, and many: longer shares, not more of them."""
import numpy as np
import pytest
import torch

from oracle import serve_oracle as orc
from serve_checks import DT, check_attention, fill_rows, num, pool, rows, seeded

pytestmark = pytest.mark.gpu

CASES = [   # lens, longest allowed, page, Hq, Hkv, D, dtype
    ([60000, 1, 0, 700, 1400] + [37] * 19, 131072, 64, 16, 8, 64, "bf16"),       # 85 shares, of 768 rows in the longest
    ([9000, 4600, 512, 513] + [3, 0] * 150, 9000, 16, 8, 8, 64, "f16"),          # seven shares
    ([2000, 300, 129, 0] * 8, 2048, 16, 4, 4, 128, "bf16"),                      # four shares, five places each
    ([400, 3, 0, 77] * 25 + [512], 512, 8, 4, 1, 128, "f16"),                    # one share, one place, a number of them that is no multiple of eight
    ([1030] * 65, 1030, 32, 2, 2, 64, "bf16"),
]


@pytest.mark.parametrize("n", range(len(CASES)))
def test_step_matches_oracle(snapkv, n):
    lens, longest, page, Hq, Hkv, D, dt = CASES[n]
    gen, dtype, B = seeded(400 + n), DT[dt], len(lens)
    q = rows(gen, B, Hq, D, dtype, "tokens")
    kp, vp, few = pool(gen, lens, page, Hkv, D, dtype)
    fill_rows(gen, kp, vp, few, lens)
    table = torch.full((B, -(-longest // page)), 1 << 30, device="cuda", dtype=torch.int32)
    table[:, :few.shape[1]] = few[:, :table.shape[1]]
    out, lse = torch.full_like(q, 77.0), torch.full((B, Hq), 77.0, device="cuda")
    ws = torch.full((snapkv.snapkv_decode_paged_workspace_bytes(B, Hq, Hkv, D, longest),), 255, dtype=torch.uint8, device="cuda")
    snapkv.snapkv_decode_attention_paged(q, kp, vp, table, torch.tensor(lens, dtype=torch.int32, device="cuda"), longest, out, lse,
                                         workspace=ws)
    torch.cuda.synchronize()
    some = np.array(lens) > 0
    assert (num(out)[~some] == 0).all() and np.isneginf(num(lse)[~some]).all()
    zero = lambda t: np.nan_to_num(num(t))
    want, want_lse, spread, reach = orc.decode_paged(num(q), zero(kp), zero(vp), table.cpu().numpy(), lens)
    check_attention(num(out)[some], num(lse)[some], want[some], want_lse[some], spread[some], reach[some], max(lens), dtype, parts=True)
