"""What a row of prompt attention does not see leaves its bits as they are, in both forms of the kernel."""
import pytest
import torch

from serve_checks import DT, offsets, rows, seeded

pytestmark = pytest.mark.gpu

# 4 heads: the keys of a row split over waves; 64 heads: whole rows to a wave
FORMS = [pytest.param(4, 2, id="split"), pytest.param(64, 32, id="whole")]


def run(snapkv, q, k, v, cu):
    T, Hq, D = q.shape
    out, lse = torch.full((T, Hq, D), 77.0, device="cuda", dtype=q.dtype), torch.full((Hq, T), 77.0, device="cuda")
    snapkv.snapkv_prompt_attention(q, k, v, cu, out, lse)
    torch.cuda.synchronize()
    return out, lse


def same(a, b, keep):
    assert torch.equal(a[1][:, keep], b[1][:, keep])
    assert torch.equal(a[0][keep], b[0][keep])


@pytest.mark.parametrize("Hq,Hkv", FORMS)
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("at", [1, 20, 31, 32, 47, 100, 300, 511, 595])
def test_a_later_key_or_value_changes_no_bit_of_an_earlier_row(snapkv, Hq, Hkv, dtype, D, at):
    """A key 50 times as long draws nearly all of the rows that see it; the 32 rows that are computed together differ in whether
    they do."""
    gen, L = seeded(1000 + at), 600
    q, k, v = (rows(gen, L, h, D, DT[dtype], "tokens") for h in (Hq, Hkv, Hkv))
    cu = offsets([L])
    want = run(snapkv, q, k, v, cu)
    before = torch.arange(L, device="cuda") < at
    k2 = k.clone()
    k2[at] *= 50
    same(run(snapkv, q, k2, v, cu), want, before)
    v2 = v.clone()
    v2[at] *= 50
    got = run(snapkv, q, k, v2, cu)
    same(got, want, before)
    assert torch.equal(got[1], want[1])


@pytest.mark.parametrize("Hq,Hkv", FORMS)
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("at", [0, 33, 300, 599])
def test_a_query_changes_no_bit_of_another_row(snapkv, Hq, Hkv, dtype, at):
    gen, L = seeded(2000 + at), 600
    q, k, v = (rows(gen, L, h, 128, DT[dtype], "tokens") for h in (Hq, Hkv, Hkv))
    cu = offsets([L])
    want = run(snapkv, q, k, v, cu)
    others = torch.arange(L, device="cuda") != at
    for what in (30.0, float("nan")):
        q2 = q.clone()
        q2[at] *= what
        same(run(snapkv, q2, k, v, cu), want, others)


@pytest.mark.parametrize("Hq,Hkv", FORMS)
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("L,at", [(1, 0), (2, 1), (33, 32), (64, 40), (100, 99), (200, 129), (595, 590)])
def test_a_later_infinity_or_nan_changes_no_bit_of_an_earlier_row(snapkv, Hq, Hkv, dtype, D, L, at):
    """In a key and in some columns of a value; rows that see them keep the other columns, a later prompt all."""
    gen = seeded(L + at)
    q, k, v = (rows(gen, L + 50, h, D, DT[dtype], "tokens") for h in (Hq, Hkv, Hkv))
    cu = offsets([L, 50])
    want = run(snapkv, q, k, v, cu)
    place = torch.arange(L + 50, device="cuda")
    before = (place < at) | (place >= L)
    some = torch.rand((Hkv, D), generator=gen, device="cuda") < 0.3
    some[:, 0] = True
    g = Hq // Hkv
    for what in (float("nan"), float("inf"), -float("inf")):
        k2, v2 = k.clone(), v.clone()
        k2[at, Hkv - 1] = what
        v2[at] = v[at].masked_fill(some, what)
        same(run(snapkv, q, k2, v2, cu), want, before)
        out, lse = run(snapkv, q, k, v2, cu)
        assert torch.equal(lse, want[1])
        same((out, lse), want, before)
        hit = some.repeat_interleave(g, 0).expand(L - at, Hq, D)
        assert not torch.isfinite(out[at:L][hit]).any()
        assert torch.equal(out[at:L][~hit], want[0][at:L][~hit])
