"""snapkv_prompt_attention against the fp64 oracle; bounds in serve_checks.py."""
import numpy as np
import pytest
import torch

from oracle import serve_oracle as orc
from serve_checks import DT, check_attention, num, offsets, rows, seeded

pytestmark = pytest.mark.gpu


def run(snapkv, q, k, v, cu, lse=True):
    T, Hq, D = q.shape
    out = torch.full((T, Hq, D), 77.0, device="cuda", dtype=q.dtype)
    out_lse = torch.full((Hq, T), 77.0, device="cuda") if lse else None
    snapkv.snapkv_prompt_attention(q, k, v, cu, out, out_lse)
    torch.cuda.synchronize()
    return out, out_lse


def check(q, k, v, cu, out, lse):
    """Rows of prompts against the oracle; the others still hold what they held."""
    want, want_lse, spread, reach = orc.prompt_attention(num(q), num(k), num(v), cu.tolist())
    mine = ~np.isnan(want_lse[0])
    n = int((cu[1:] - cu[:-1]).max())
    got, got_lse = num(out), num(lse) if lse is not None else None
    assert (got[~mine] == 77).all()
    if lse is not None:
        assert (got_lse[:, ~mine] == 77).all()
    check_attention(got[mine], got_lse[:, mine].T if lse is not None else None, want[mine], want_lse[:, mine].T, spread[mine],
                    reach[:, mine].T, n, q.dtype, parts=False)


LENGTHS = [[1], [2], [1, 1, 1], [31, 32, 33], [63, 64, 65], [127, 128, 129, 0, 255, 256, 257], [0, 5, 0], [700], [1025, 3], [17] * 70,
           [1] * 200, [511, 512, 513], [0, 200, 1, 0, 33, 129] * 13, [7] * 64 + [0] * 70 + [300]]


@pytest.mark.parametrize("lengths", LENGTHS, ids=lambda x: "x".join(map(str, x[:7])))
@pytest.mark.parametrize("D", [64, 128])
def test_lengths(snapkv, lengths, D):
    gen, T = seeded(sum(lengths) + D), sum(lengths)
    q, k, v = (rows(gen, T, h, D, torch.bfloat16, "fused") for h in (4, 2, 2))
    cu = offsets(lengths)
    out, lse = run(snapkv, q, k, v, cu)
    check(q, k, v, cu, out, lse)


@pytest.mark.parametrize("lengths", [[1025, 3], [511, 512, 513], [127, 128, 129, 0, 255, 256, 257], [0, 200, 1, 0, 33, 129] * 13], ids=lambda x: "x".join(map(str, x[:7])))
@pytest.mark.parametrize("D", [64, 128])
def test_lengths_of_many_heads(snapkv, lengths, D):
    """Whole rows to a wave: the form of calls that fill the chip (the ones above split the keys of a row over waves)."""
    gen, T = seeded(sum(lengths) + D), sum(lengths)
    q, k, v = (rows(gen, T, h, D, torch.float16, "fused") for h in (48, 16, 16))
    cu = offsets(lengths)
    out, lse = run(snapkv, q, k, v, cu)
    check(q, k, v, cu, out, lse)


def test_both_forms_agree(snapkv):
    """The same heads alone (keys split) and among others (whole rows): equal up to rounding, also behind NaN values."""
    gen, L = seeded(40), 1100
    q, k, v = (rows(gen, L, h, 128, torch.bfloat16, "tokens") for h in (40, 40, 40))
    v[700:, :, ::3] = float("nan")
    cu = offsets([L])
    wide, wide_lse = run(snapkv, q, k, v, cu)
    some = [t[:, 8:12].contiguous() for t in (q, k, v)]
    out, lse = run(snapkv, *some, cu)
    assert (lse - wide_lse[8:12]).abs().max() <= 1e-5
    a, b = out.float(), wide[:, 8:12].float()
    assert torch.equal(torch.isnan(a), torch.isnan(b)) and torch.isfinite(a[:700]).all() and torch.isnan(a[700:, :, ::3]).all()
    # each within two roundings of the exact value: probabilities (of mean |v|) and the result
    near = 2 * 2.0 ** -8 * (b.nan_to_num().abs() + float(v[:700].float().abs().mean())) + 1e-4
    assert ((a - b).nan_to_num().abs() <= near).all()


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (8, 8), (7, 1), (6, 3), (12, 12), (16, 4), (10, 5), (32, 8), (24, 24), (20, 2)])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_heads(snapkv, Hq, Hkv, dtype):
    gen = seeded(Hq * 100 + Hkv)
    lengths = [150, 1, 301]
    q, k, v = (rows(gen, sum(lengths), h, 128, DT[dtype], "tokens") for h in (Hq, Hkv, Hkv))
    cu = offsets(lengths)
    out, lse = run(snapkv, q, k, v, cu)
    check(q, k, v, cu, out, lse)


@pytest.mark.parametrize("layouts", [("heads", "heads", "heads"), ("tokens", "fused", "heads"), ("fused", "heads", "tokens")])
@pytest.mark.parametrize("D", [64, 128])
def test_storage_orders(snapkv, layouts, D):
    gen = seeded(D)
    lengths = [97, 260]
    q, k, v = (rows(gen, sum(lengths), h, D, torch.float16, x) for h, x in zip((6, 3, 3), layouts))
    cu = offsets(lengths)
    out, lse = run(snapkv, q, k, v, cu)
    check(q, k, v, cu, out, lse)
    again, _ = run(snapkv, q.contiguous(), k.contiguous(), v.contiguous(), cu, lse=False)      # the same bits, and no lse asked for
    assert torch.equal(out, again)


@pytest.mark.parametrize("Hq,Hkv", [(32, 8), (64, 64)])
def test_many_prompts_fill_the_chip(snapkv, Hq, Hkv):
    """Enough row tiles for the form that large calls take."""
    gen = seeded(Hq)
    lengths = [300, 1, 257, 777, 64, 513, 255]
    q, k, v = (rows(gen, sum(lengths), h, 64, torch.bfloat16, "fused") for h in (Hq, Hkv, Hkv))
    cu = offsets(lengths)
    out, lse = run(snapkv, q, k, v, cu)
    check(q, k, v, cu, out, lse)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("kind", ["sharp", "flat", "falling", "rising", "shifted"])
def test_distributions(snapkv, dtype, kind):
    """One key takes all; all alike; the largest logits first or last (the running maximum moves every tile); large sums."""
    gen, L = seeded(5), 600
    q, k, v = (rows(gen, L, h, 128, DT[dtype], "tokens") for h in (4, 2, 2))
    if kind == "sharp":
        q.mul_(12)
    elif kind == "flat":
        q.zero_()
    elif kind in ("falling", "rising"):
        ramp = torch.linspace(0, 4, L, device="cuda") if kind == "rising" else torch.linspace(4, 0, L, device="cuda")
        q.copy_((1 + 0.1 * q.float()).to(q.dtype))
        k.copy_((ramp[:, None, None] + 0.1 * k.float()).to(k.dtype))
    else:
        k.add_(6)
        v.add_(3)
    cu = offsets([L])
    out, lse = run(snapkv, q, k, v, cu)
    check(q, k, v, cu, out, lse)


@pytest.mark.parametrize("first,last", [(0, 33), (41, 0), (64, 64)])
def test_rows_of_no_prompt_are_neither_read_nor_written(snapkv, first, last):
    gen, lengths = seeded(6), [70, 130]
    T = first + sum(lengths) + last
    q, k, v = (rows(gen, T, h, 128, torch.bfloat16, "tokens") for h in (4, 2, 2))
    for t in (q, k, v):
        t[:first] = float("nan")
        t[T - last:] = float("inf")
    cu = offsets(lengths, first)
    out, lse = run(snapkv, q, k, v, cu)
    a, e = first, T - last
    assert (out[:a] == 77).all() and (out[e:] == 77).all() and (lse[:, :a] == 77).all() and (lse[:, e:] == 77).all()
    check(q[a:e], k[a:e], v[a:e], cu - first, out[a:e], lse[:, a:e])


def test_thousands_of_prompts(snapkv):
    """Lengths of 0 to 140 of 4500 prompts behind tokens of none: every one found, none twice."""
    gen = seeded(60)
    lengths = (torch.randint(0, 71, (4500,), generator=gen, device="cuda") * (1 + torch.randint(0, 2, (4500,), generator=gen, device="cuda"))).tolist()
    T = 999 + sum(lengths) + 50
    q, k, v = (rows(gen, T, h, 64, torch.bfloat16, "tokens") for h in (2, 1, 1))
    cu = offsets(lengths, 999)
    out, lse = run(snapkv, q, k, v, cu)
    assert (out[:999] == 77).all() and (out[T - 50:] == 77).all() and (lse[:, :999] == 77).all() and (lse[:, T - 50:] == 77).all()
    at = cu.tolist()
    for some in (range(0, 130), range(2200, 2230), range(4400, 4500)):
        a, e = at[some[0]], at[some[-1] + 1]
        check(q[a:e], k[a:e], v[a:e], cu[some[0]:some[-1] + 2] - a, out[a:e], lse[:, a:e])
    assert torch.isfinite(out).all() and not (lse[:, 999:T - 50] == 77).any()


def test_a_prompt_does_not_see_its_neighbours(snapkv):
    gen = seeded(7)
    q, k, v = (rows(gen, 400, h, 64, torch.float16, "tokens") for h in (2, 1, 1))
    cu = offsets([100, 200, 100])
    out, lse = run(snapkv, q, k, v, cu)
    for t in (q, k, v):
        t[:100] = float("nan")
        t[300:] = float("nan")
    again, again_lse = run(snapkv, q, k, v, cu)
    assert torch.equal(out[100:300], again[100:300]) and torch.equal(lse[:, 100:300], again_lse[:, 100:300])


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("L,at", [(1, 0), (2, 1), (33, 32), (64, 40), (100, 99), (200, 129), (300, 297)])
def test_values_that_a_row_does_not_see_may_be_anything(snapkv, dtype, D, L, at):
    """Infinities and NaN in a later token's key and value reach no earlier row; a later prompt starts anew."""
    gen = seeded(L + at)
    q, k, v = (rows(gen, L + 50, h, D, DT[dtype], "tokens") for h in (4, 2, 2))
    cu = offsets([L, 50])
    want, want_lse = run(snapkv, q, k, v, cu)
    for what in (float("nan"), float("inf"), -float("inf")):
        k2, v2 = k.clone(), v.clone()
        k2[at, 1] = what
        v2[at] = torch.where(torch.rand((2, D), generator=gen, device="cuda") < 0.3, what, v[at].float()).to(v.dtype)
        v2[at, :, 0] = what
        out, lse = run(snapkv, q, k2, v2, cu)
        keep = torch.ones(L + 50, dtype=torch.bool, device="cuda")
        keep[at:L] = False
        assert torch.equal(lse[:, keep], want_lse[:, keep])
        # (values added one by one may round otherwise than sixteen at a time: one step of the type at most)
        assert ((out[keep].float() - want[keep].float()).abs() <= torch.finfo(DT[dtype]).eps * want[keep].float().abs() + 1e-5).all()
        assert not torch.isfinite(out[at]).all()


def test_keys_of_minus_infinity_take_no_part(snapkv):
    """Logits of -infinity over the first blocks of a row: their probability is 0, whatever comes later."""
    gen, L = seeded(77), 150
    q, k, v = (rows(gen, L, h, 64, torch.bfloat16, "tokens") for h in (2, 1, 1))
    q.copy_(q.abs() + 0.1)
    k[:70] = -float("inf")
    cu = offsets([L])
    out, lse = run(snapkv, q, k, v, cu)
    assert torch.isnan(out[:70]).all() and torch.isneginf(lse[:, :70]).all()         # (nothing to average)
    for i in (70, 71, 96, 127, 128, 149):
        for h in range(2):
            s = k[70:i + 1, 0].double() @ q[i, h].double() / 8.0
            z = torch.logsumexp(s, 0)
            p = (s - z).exp()
            reach = (k[70:i + 1, 0].double().abs() @ q[i, h].double().abs()).max() / 8.0
            check_attention(num(out[i, h])[None], num(lse[h, i])[None], num(p @ v[70:i + 1, 0].double())[None], num(z)[None],
                            num(p @ v[70:i + 1, 0].double().abs())[None], num(reach)[None], L, torch.bfloat16, parts=False)


def test_offsets_outside_the_tensors_are_clamped(snapkv):
    gen = seeded(8)
    q, k, v = (rows(gen, 150, h, 64, torch.bfloat16, "tokens") for h in (2, 2, 2))
    out, lse = run(snapkv, q, k, v, torch.tensor([-7, 60, 40, 1 << 30], dtype=torch.int32, device="cuda"))
    # prompts [0, 60) and [40, 150); rows 40 .. 59 are either's
    for (a, e), mine in (((0, 60), slice(0, 40)), ((40, 150), slice(60, 150))):
        want, want_lse, spread, reach = orc.prompt_attention(num(q), num(k), num(v), [a, e])
        check_attention(num(out)[mine], num(lse)[:, mine].T, want[mine], want_lse[:, mine].T, spread[mine], reach[:, mine].T, e - a, q.dtype, parts=False)
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()


def test_rows_beyond_32_bit_offsets(snapkv):
    """Rows of a tensor of more than 2^31 elements."""
    T, H, D = 300, 2, 128
    wide = torch.empty((T, 1 << 23), device="cuda", dtype=torch.bfloat16)
    q, k, v = (wide[:, c:c + H * D].view(T, H, D) for c in (0, 1024, 1 << 22))
    for i, t in enumerate((q, k, v)):
        t.copy_(torch.randn((T, H, D), generator=seeded(20 + i), device="cuda"))
    cu = offsets([T])
    out, lse = run(snapkv, q, k, v, cu)
    again, again_lse = run(snapkv, q.contiguous(), k.contiguous(), v.contiguous(), cu)
    assert torch.equal(out, again) and torch.equal(lse, again_lse)
    check(q.contiguous(), k.contiguous(), v.contiguous(), cu, out, lse)


def test_long_prompt_by_samples(snapkv):
    """Rows of a prompt of 20011 tokens against float64 on the device."""
    gen, L, D = seeded(9), 20011, 128
    q, k, v = (rows(gen, L, h, D, torch.bfloat16, "fused") for h in (4, 1, 1))
    out, lse = run(snapkv, q, k, v, offsets([L]))
    kd, vd = k[:, 0].double(), v[:, 0].double()
    for i in (0, 63, 64, 9999, 16384, 20000, L - 1):
        for h in range(4):
            qd = q[i, h].double()
            s = kd[:i + 1] @ qd / D ** 0.5
            z = torch.logsumexp(s, 0)
            p = (s - z).exp()
            reach = (kd[:i + 1].abs() @ qd.abs()).max() / D ** 0.5
            check_attention(num(out[i, h])[None], num(lse[h, i])[None], num(p @ vd[:i + 1])[None], num(z)[None],
                            num(p @ vd[:i + 1].abs())[None], num(reach)[None], i + 1, torch.bfloat16, parts=False)


def test_calls_repeat_bit_for_bit_and_a_captured_one_follows_its_offsets(snapkv):
    gen = seeded(10)
    q, k, v = (rows(gen, 900, h, 128, torch.bfloat16, "fused") for h in (8, 4, 4))
    cu, out, lse = offsets([300, 600]), torch.zeros((900, 8, 128), device="cuda", dtype=torch.bfloat16), torch.zeros((8, 900), device="cuda")
    graph = torch.cuda.CUDAGraph()
    snapkv.snapkv_prompt_attention(q, k, v, cu, out, lse)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        snapkv.snapkv_prompt_attention(q, k, v, cu, out, lse)
    for lengths in ([300, 600], [1, 899], [500, 0], [450, 450]):
        cu.copy_(offsets(lengths))
        q.normal_(generator=gen)
        out.fill_(77), lse.fill_(77)
        want = run(snapkv, q, k, v, cu)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


def test_calls_on_two_streams_are_independent(snapkv):
    sets = []
    for s in range(2):
        gen = seeded(30 + s)
        sets.append([rows(gen, 1200, h, 64, torch.float16, "tokens") for h in (8, 8, 8)] + [offsets([700, 500])])
    want = [run(snapkv, *x) for x in sets]
    streams, got = [torch.cuda.Stream() for _ in sets], [[], []]
    for _ in range(8):
        for x, st, g in zip(sets, streams, got):
            o, l = torch.empty_like(want[0][0]), torch.empty_like(want[0][1])
            st.wait_stream(torch.cuda.current_stream())
            snapkv.snapkv_prompt_attention(*x, o, l, stream=st)
            g.append((o, l))
    torch.cuda.synchronize()
    for w, g in zip(want, got):
        assert all(torch.equal(o, w[0]) and torch.equal(l, w[1]) for o, l in g)
