"""A mean of finite values is finite: the rounding of probabilities must not carry it past the type's largest number."""
import numpy as np
import pytest
import torch

from serve_checks import check_attention, num, offsets

L, D, BIG = 300, 64, 65504.0
Q0, K0 = 8.2890625, -0.66845703125       # exp(Q0 K0 / 8) = 0.50027, which fp16 rounds up by 0.00044 of it


def probabilities():
    """Every 32nd key has logit 0, the others the one above; row i sees keys 0 .. i."""
    p = np.where(np.arange(L) % 32 == 0, 1.0, np.exp(Q0 * K0 / 8))
    return p, p.astype(np.float16).astype(np.float64)


def test_the_probabilities_round_up():
    """(that these inputs do reach past the largest number: 65520 and more round to infinity)"""
    p, rounded = probabilities()
    mean = BIG * rounded.cumsum() / p.cumsum()
    assert (mean[40:] > 65522).all()


@pytest.mark.gpu
@pytest.mark.parametrize("Hq", [4, 512], ids=["split", "whole"])
def test_a_mean_of_the_largest_numbers_is_one(snapkv, Hq):
    q = torch.zeros((L, Hq, D), device="cuda", dtype=torch.float16)
    q[:, :, 0] = Q0
    k = torch.zeros((L, Hq, D), device="cuda", dtype=torch.float16)
    k[:, :, 0] = K0
    k[::32] = 0
    v = torch.full((L, Hq, D), BIG, device="cuda", dtype=torch.float16)
    v[:, :, ::3] = -BIG
    v[:, :, 1] = 1.0
    out, lse = torch.empty_like(q), torch.empty((Hq, L), device="cuda")
    cu = offsets([L])
    snapkv.snapkv_prompt_attention(q, k, v, cu, out, lse)
    torch.cuda.synchronize()
    want = num(v)
    p, _ = probabilities()
    reach = np.full((L, Hq), abs(Q0 * K0) / 8)
    check_attention(num(out), num(lse).T, want, np.log(p.cumsum())[:, None].repeat(Hq, 1), np.abs(want), reach, L, torch.float16, parts=False)
    v[5:, :, 2] = float("inf")                       # an infinity stays one
    v[5:, :, 3] = -float("inf")
    snapkv.snapkv_prompt_attention(q, k, v, cu, out, lse)
    torch.cuda.synchronize()
    assert torch.isposinf(out[5:, :, 2]).all() and torch.isneginf(out[5:, :, 3]).all() and torch.isfinite(out[:5]).all()
    assert torch.isfinite(out[:, :, 4:]).all()
