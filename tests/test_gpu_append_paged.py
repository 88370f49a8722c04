"""snapkv_append_paged against the fp64 oracle; bounds in serve_checks.py."""
import numpy as np
import pytest
import torch

from oracle import serve_oracle as orc
from serve_checks import DT, W24, half_step, num, offsets, pool, rows, seeded, tables

pytestmark = pytest.mark.gpu


def close(got, want, a_plus_b, dtype):
    err, bound = np.abs(num(got) - want), half_step(dtype) * np.abs(want) + 4 * W24 * a_plus_b + 1e-38
    if dtype == torch.float16:
        bound = bound + 2.0 ** -25          # half a step of fp16's smallest numbers
    assert (err <= bound).all(), float((err / bound).max())


def partners(x, half, interleaved):
    """|a| + |b| of the pair that each element belongs to (0 where nothing is turned)."""
    y = np.zeros_like(x)
    for m in range(half):
        i, j = (2 * m, 2 * m + 1) if interleaved else (m, m + half)
        y[..., i] = y[..., j] = np.abs(x[..., i]) + np.abs(x[..., j])
    return y


def bits(t):
    return t.contiguous().view(torch.int32 if t.element_size() == 4 else torch.int16)


CASES = [   # lengths, starts, page, Hq, Hkv, D, dtype, rot, interleaved, layout, queries, keys out
    ([1] * 8, [5, 0, 16, 15, 17, 100, 31, 32], 16, 32, 8, 128, "bf16", 128, False, "fused", True, False),
    ([1], [0], 1, 1, 1, 64, "f32", 64, True, "tokens", True, True),
    ([3, 0, 70, 1], [0, 9, 13, 40], 7, 6, 2, 64, "f16", 32, False, "heads", True, True),
    ([33, 64, 1], [0, 0, 0], 32, 8, 8, 128, "bf16", 64, True, "fused", True, True),
    ([130], [3], 24, 0, 4, 128, "f16", 0, False, "heads", False, False),
    ([40, 41], [0, 1], 8, 12, 4, 128, "f32", 128, False, "fused", True, False),
    ([9, 5], [2, 2], 16, 0, 3, 64, "bf16", 48, True, "tokens", False, True),
    ([700, 1, 500], [0, 2047, 77], 64, 4, 1, 128, "bf16", 128, False, "tokens", True, True),
    ([1] * 131, list(range(131)), 16, 2, 1, 64, "bf16", 64, False, "fused", True, False),      # sequences of three searches
]


@pytest.mark.parametrize("n", range(len(CASES)))
def test_append_matches_oracle(snapkv, n):
    lengths, starts, page, Hq, Hkv, D, dt, rot, interleaved, layout, queries, keys_out = CASES[n]
    dtype, gen, T, B = DT[dt], seeded(100 + n), sum(lengths), len(lengths)
    k, v = (rows(gen, T, Hkv, D, dtype, layout) for _ in range(2))
    q = rows(gen, T, Hq, D, dtype, layout) if queries else None
    kp, vp, table = pool(gen, [a + m for a, m in zip(starts, lengths)], page, Hkv, D, dtype, fill=7.0)
    P = max(a + m for a, m in zip(starts, lengths)) + 50
    cos, sin = tables(P, rot // 2) if rot else (None, None)
    pos = torch.randint(0, P, (T,), generator=gen, device="cuda").to(torch.int32) if rot else None
    q_out = rows(gen, T, Hq, D, dtype, layout) if queries else None
    k_out = rows(gen, T, Hkv, D, dtype, layout) if keys_out else None
    cu, st = offsets(lengths), torch.tensor(starts, dtype=torch.int32, device="cuda")
    old_k, old_v = num(kp), num(vp)
    snapkv.snapkv_append_paged(k, v, kp, vp, table, st, cu_seqlens=cu, positions=pos, cos=cos, sin=sin, interleaved=interleaved,
                               q=q, q_out=q_out, k_out=k_out)
    torch.cuda.synchronize()
    turn = lambda x: orc.rotate(num(x), pos.tolist(), num(cos), num(sin), interleaved) if rot else num(x)
    size = lambda x: partners(num(x), rot // 2, interleaved)
    want_k, want_v = orc.append(old_k, old_v, turn(k), num(v), table.cpu().numpy(), starts, cu.tolist())
    size_k, _ = orc.append(0 * old_k, 0 * old_v, size(k), num(v), table.cpu().numpy(), starts, cu.tolist())
    close(kp, want_k, size_k, dtype)
    assert np.array_equal(num(vp), want_v)                    # copied, and everything else as it was
    if not rot:
        assert np.array_equal(num(kp), want_k)
    if queries:
        close(q_out, turn(q), size(q), dtype)
    if keys_out:
        close(k_out, turn(k), size(k), dtype)
        for b in range(B):                                    # the same numbers in both places
            for t in range(int(cu[b]), int(cu[b + 1])):
                r = starts[b] + t - int(cu[b])
                assert torch.equal(bits(kp[int(table[b, r // page]), r % page]), bits(k_out[t]))


def test_rows_without_a_page_and_tokens_of_no_sequence_are_left_alone(snapkv):
    gen = seeded(7)
    k, v, q = rows(gen, 12, 2, 64, torch.bfloat16, "tokens"), rows(gen, 12, 2, 64, torch.bfloat16, "tokens"), rows(gen, 12, 4, 64, torch.bfloat16, "tokens")
    kp = torch.zeros((4, 4, 2, 64), device="cuda", dtype=torch.bfloat16)
    vp = torch.zeros_like(kp)
    table = torch.tensor([[1, -1], [9, 2]], dtype=torch.int32, device="cuda")
    cu, st = torch.tensor([2, 7, 10], dtype=torch.int32, device="cuda"), torch.tensor([2, 6], dtype=torch.int32, device="cuda")
    cos, sin = tables(16, 32)
    q_out, k_out = torch.full_like(q, 9.0), torch.full_like(k, 9.0)
    snapkv.snapkv_append_paged(k, v, kp, vp, table, st, cu_seqlens=cu, cos=cos, sin=sin, q=q, q_out=q_out, k_out=k_out)
    torch.cuda.synchronize()
    # rows 2, 3 of the first sequence have page 1, its rows 4-6 no page; the second's rows 6, 7 page 2, its row 8 no column
    want_k, want_v = orc.append(np.zeros(kp.shape), np.zeros(kp.shape), num(k_out), num(v), table.cpu().numpy(), [2, 6], cu.tolist())
    assert np.array_equal(num(kp), want_k) and np.array_equal(num(vp), want_v)
    assert (vp.flatten(1).abs().sum(1) > 0).tolist() == [False, True, True, False]
    for t in (0, 1, 10, 11):
        assert (q_out[t] == 9).all() and (k_out[t] == 9).all()
    pos = [0, 0, 2, 3, 4, 5, 6, 6, 7, 8]                     # without positions a token's row is its position
    close(q_out[2:10], orc.rotate(num(q)[:10], pos, num(cos), num(sin), False)[2:], partners(num(q)[2:10], 32, False), torch.bfloat16)


def test_one_token_each_needs_no_offsets_and_positions_are_clamped(snapkv):
    gen, B = seeded(8), 5
    k, v = rows(gen, B, 2, 128, torch.float16, "heads"), rows(gen, B, 2, 128, torch.float16, "fused")
    st = torch.tensor([0, 3, 4, 7, 8], dtype=torch.int32, device="cuda")
    cos, sin = tables(20, 64)
    pos = torch.tensor([-4, 0, 19, 20, 1 << 30], dtype=torch.int32, device="cuda")
    got = []
    for cu in (None, offsets([1] * B)):
        kp, vp, table = pool(seeded(9), [9] * B, 4, 2, 128, torch.float16, fill=0.0)
        k_out = torch.empty_like(k)
        snapkv.snapkv_append_paged(k, v, kp, vp, table, st, cu_seqlens=cu, positions=pos, cos=cos, sin=sin, k_out=k_out)
        torch.cuda.synchronize()
        got.append((kp, vp, k_out))
    assert all(torch.equal(a, b) for a, b in zip(*got))
    close(got[0][2], orc.rotate(num(k), pos.tolist(), num(cos), num(sin), False), partners(num(k), 64, False), torch.float16)


def test_pages_and_rows_beyond_32_bit_offsets(snapkv):
    """More than 2^31 elements in the pool and between a row and the first."""
    page, Hkv, D = 128, 8, 128
    pages = (1 << 31) // (page * Hkv * D) + 40
    kp = torch.empty((pages, page, Hkv, D), device="cuda", dtype=torch.bfloat16)
    vp = torch.empty_like(kp)
    wide = torch.empty((3, (1 << 30) + 1024), device="cuda", dtype=torch.bfloat16)
    k = wide[:, :Hkv * D].view(3, Hkv, D).copy_(torch.randn((3, Hkv, D), generator=seeded(10), device="cuda"))
    table = torch.tensor([[0, pages - 1]], dtype=torch.int32, device="cuda")
    st = torch.tensor([page - 1], dtype=torch.int32, device="cuda")
    k_out = wide[:, 4096:4096 + Hkv * D].view(3, Hkv, D)
    snapkv.snapkv_append_paged(k, k, kp, vp, table, st, cu_seqlens=offsets([3]), k_out=k_out)
    torch.cuda.synchronize()
    for p in (kp, vp):
        assert torch.equal(p[0, page - 1], k[0]) and torch.equal(p[pages - 1, 0], k[1]) and torch.equal(p[pages - 1, 1], k[2])
    assert torch.equal(k_out, k)


def test_captured_call_follows_its_inputs(snapkv):
    """Offsets, starts, positions and tables are read on the device: a replay goes by what they hold then."""
    gen = seeded(11)
    k, v, q = (rows(gen, 40, h, 64, torch.bfloat16, "tokens") for h in (2, 2, 4))
    cos, sin = tables(600, 32)
    q_out, k_out = torch.empty_like(q), torch.empty_like(k)
    cu, st = offsets([10, 30]), torch.tensor([0, 0], dtype=torch.int32, device="cuda")
    pos = torch.arange(40, device="cuda", dtype=torch.int32)
    kp, vp, table = pool(gen, [64, 64], 16, 2, 64, torch.bfloat16, fill=0.0)
    call = lambda a, b, c, d: snapkv.snapkv_append_paged(k, v, a, b, table, st, cu_seqlens=cu, positions=pos, cos=cos, sin=sin,
                                                         q=q, q_out=c, k_out=d)
    call(kp, vp, q_out, k_out)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        call(kp, vp, q_out, k_out)
    for rep, (lengths, starts) in enumerate([([10, 30], [0, 0]), ([1, 20], [33, 9]), ([0, 40], [5, 24]), ([25, 15], [7, 30])]):
        cu.copy_(offsets(lengths))
        st.copy_(torch.tensor(starts))
        pos.copy_(torch.randint(0, 600, (40,), generator=gen, device="cuda"))
        k.normal_(generator=gen)
        for t in (kp, vp, q_out, k_out):
            t.zero_()
        want = [torch.zeros_like(t) for t in (kp, vp, q_out, k_out)]
        call(*want)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (kp, vp, q_out, k_out))), rep
        assert kp.any()
