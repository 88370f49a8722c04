"""The step over pages where numbers are small, or no numbers."""
import numpy as np
import pytest
import torch

from oracle import serve_oracle as orc
from serve_checks import DT, check_attention, fill_rows, num, pool, rows, seeded

pytestmark = pytest.mark.gpu

LENGTHS = [pytest.param([500, 40], id="whole"), pytest.param([3000, 129], id="split")]


def run(snapkv, q, kp, vp, table, lens):
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    snapkv.snapkv_decode_attention_paged(q, kp, vp, table, torch.tensor(lens, dtype=torch.int32, device="cuda"), max(lens), out, lse)
    torch.cuda.synchronize()
    return out, lse


@pytest.mark.parametrize("lens", LENGTHS)
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_a_query_that_is_no_number_has_no_answer(snapkv, lens, dtype):
    """NaN in one head's query (a zero would pass for an answer); the other heads as before.  Logits of plus infinity likewise."""
    gen = seeded(31)
    q = rows(gen, 2, 8, 128, DT[dtype], "tokens")
    kp, vp, table = pool(gen, lens, 16, 2, 128, DT[dtype])
    fill_rows(gen, kp, vp, table, lens)
    want = run(snapkv, q, kp, vp, table, lens)
    others = torch.ones((2, 8), dtype=torch.bool, device="cuda")
    others[0, 5] = others[1, 2] = False
    for what in (float("nan"), float("inf")):
        q2 = q.clone()
        q2[0, 5, 77] = q2[1, 2, 0] = what
        out, lse = run(snapkv, q2, kp, vp, table, lens)
        assert torch.isnan(out[~others]).all() and torch.isnan(lse[~others]).all()
        assert torch.equal(out[others], want[0][others]) and torch.equal(lse[others], want[1][others])
