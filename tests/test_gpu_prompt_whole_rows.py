"""The form of prompt attention that gives whole rows to a wave, where other tests meet the one that splits their keys."""
import numpy as np
import pytest
import torch

from serve_checks import DT, check_attention, num, offsets, rows, seeded

pytestmark = pytest.mark.gpu


def run(snapkv, q, k, v, cu):
    out, lse = torch.full(q.shape, 77.0, device="cuda", dtype=q.dtype), torch.full((q.shape[1], q.shape[0]), 77.0, device="cuda")
    snapkv.snapkv_prompt_attention(q, k, v, cu, out, lse)
    torch.cuda.synchronize()
    return out, lse


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_rows_beyond_32_bit_offsets(snapkv, D, dtype):
    """Rows 2^24 elements apart, of a tensor of more than 2^31, in prompts of several tiles and of less than one."""
    lengths = [200, 3, 64]
    T, H = sum(lengths), 64
    wide = torch.empty((T, 1 << 24), device="cuda", dtype=DT[dtype])
    q, k, v = (wide[:, c:c + H * D].view(T, H, D) for c in (0, 1 << 20, 1 << 23))
    for i, t in enumerate((q, k, v)):
        t.copy_(torch.randn((T, H, D), generator=seeded(20 + i), device="cuda"))
    cu = offsets(lengths)
    out, lse = run(snapkv, q, k, v, cu)
    again, again_lse = run(snapkv, q.contiguous(), k.contiguous(), v.contiguous(), cu)
    assert torch.equal(out, again) and torch.equal(lse, again_lse)
    at = 0
    for n in lengths:
        some = slice(at, at + n)
        s = torch.matmul(q[some].double().permute(1, 0, 2).contiguous(), k[some].double().permute(1, 2, 0).contiguous()) / D ** 0.5
        s.masked_fill_(torch.ones((n, n), dtype=torch.bool, device="cuda").triu(1), -float("inf"))
        p = torch.softmax(s, -1)
        vd = v[some].double().transpose(0, 1).contiguous()
        reach = torch.matmul(q[some].double().abs().permute(1, 0, 2).contiguous(), k[some].double().abs().permute(1, 2, 0).contiguous()) / D ** 0.5
        check_attention(num(out[some].transpose(0, 1)), num(lse[:, some]), num(torch.matmul(p, vd)), num(torch.logsumexp(s, -1)),
                        num(torch.matmul(p, vd.abs())), num(reach.tril().amax(-1)), n, DT[dtype], parts=False)
        at += n


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_keys_of_minus_infinity_take_no_part(snapkv, D, dtype):
    """Logits of -infinity over the first blocks of a row: their probability is 0, whatever comes later."""
    gen, L, H = seeded(78), 300, 64
    q, k, v = (rows(gen, L, h, D, DT[dtype], "tokens") for h in (H, H // 2, H // 2))
    q.copy_(q.abs() + 0.1)
    k[:170] = -float("inf")
    out, lse = run(snapkv, q, k, v, offsets([L]))
    assert torch.isnan(out[:170]).all() and torch.isneginf(lse[:, :170]).all()       # (nothing to average)
    for i in (170, 171, 191, 192, 255, 256, 299):
        for h in (0, 33, 63):
            s = k[170:i + 1, h // 2].double() @ q[i, h].double() / D ** 0.5
            z = torch.logsumexp(s, 0)
            p = (s - z).exp()
            vd = v[170:i + 1, h // 2].double()
            reach = (k[170:i + 1, h // 2].double().abs() @ q[i, h].double().abs()).max() / D ** 0.5
            check_attention(num(out[i, h])[None], num(lse[h, i])[None], num(p @ vd)[None], num(z)[None], num(p @ vd.abs())[None],
                            num(reach)[None], L, DT[dtype], parts=False)
