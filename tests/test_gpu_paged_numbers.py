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


@pytest.mark.parametrize("lens", LENGTHS + [pytest.param([70000], id="long")])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("D", [64, 128])
def test_many_small_probabilities_count_as_much_as_one(snapkv, lens, dtype, D):
    """The first row takes most of the probability and holds zeros, so that all of the answer comes from rows of about 2^-17 of its
    probability each: below fp16's normal numbers."""
    gen, Hq, Hkv = seeded(32), 8, 2
    q = torch.zeros((len(lens), Hq, D), device="cuda", dtype=DT[dtype])
    q[:, :, 0] = D ** 0.5
    kp, vp, table = pool(gen, lens, 16, Hkv, D, DT[dtype])
    fill_rows(gen, kp, vp, table, lens)
    for t in (kp, vp):
        t.nan_to_num_(0.0)
    kp[..., 0] = kp[..., 0] * 0.25 - 11.8
    vp.abs_()
    first = table[:, 0].long()
    kp[first, 0] = 0
    vp[first, 0] = 0
    out, lse = run(snapkv, q, kp, vp, table, lens)
    want, want_lse, spread, reach = orc.decode_paged(num(q), num(kp), num(vp), table.cpu().numpy(), lens)
    check_attention(num(out), num(lse), want, want_lse, spread, reach, max(lens), DT[dtype], parts=True)
