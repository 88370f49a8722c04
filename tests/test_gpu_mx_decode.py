"""snapkv_decode_attention_paged_mx against the fp64 oracle; bounds in mx_checks.py."""
import numpy as np
import pytest
import torch

from mx_checks import check_step, mx_pool, mx_values
from oracle import serve_oracle as orc
from serve_checks import DT, num, rows, seeded

pytestmark = pytest.mark.gpu


def run(snapkv, q, pool, table, lens, max_len, lse=True, **kw):
    out = torch.full(q.shape, 77.0, device="cuda", dtype=q.dtype)
    out_lse = torch.full(q.shape[:2], 77.0, device="cuda") if lse else None
    snapkv.snapkv_decode_attention_paged_mx(q, *pool, table, lens, max_len, out, out_lse, **kw)
    return out, out_lse


def check(q, pool, kind, table, lens, out, lse):
    torch.cuda.synchronize()
    want = orc.decode_paged(num(q), mx_values(pool[0], pool[1], kind), mx_values(pool[2], pool[3], kind), table.cpu().numpy(), lens)
    check_step(out, lse, *want, max(max(lens), 1), q.dtype)


CASES = [   # lens, page, Hq, Hkv, D, dtype, room beyond the longest
    ([1], 16, 4, 4, 128, "bf16", 0),
    ([0, 1, 15, 16, 17, 31, 32, 33], 16, 8, 2, 64, "bf16", 5),
    ([127, 128, 129, 255, 256, 257], 8, 16, 1, 128, "f16", 0),
    ([511, 512, 513, 1], 32, 32, 8, 128, "bf16", 0),
    ([2113], 16, 32, 8, 128, "f16", 400),
    ([4097, 3], 24, 3, 3, 64, "f16", 0),
    ([1000, 7, 0, 2500], 1, 6, 2, 128, "bf16", 0),
    ([300, 301], 7, 10, 5, 64, "bf16", 1),
    ([20000], 64, 4, 2, 64, "bf16", 0),
    ([900, 1], 128, 24, 24, 128, "bf16", 31000),
    ([64] * 150, 16, 2, 2, 64, "f16", 0),
    ([5000, 1, 777, 0, 4096, 130, 129], 16, 8, 4, 128, "bf16", 0),
    ([3000] + [1] * 40, 16, 4, 2, 64, "bf16", 20000),
]


@pytest.mark.parametrize("kind", ["fp8", "fp4"])
@pytest.mark.parametrize("n", range(len(CASES)))
def test_step_matches_oracle(snapkv, n, kind):
    lens, page, Hq, Hkv, D, dt, room = CASES[n]
    gen = seeded(1200 + n)
    q = rows(gen, len(lens), Hq, D, DT[dt], "tokens")
    pool, table = mx_pool(gen, [x + room for x in lens], page, Hkv, D, kind)
    for s in (pool[1], pool[3]):                                   # rows behind a sequence's own are never read
        for b, x in enumerate(lens):
            j = torch.arange(x, x + room, device="cuda")
            s[table[b, j // page].long(), j % page] = 255
    dl = torch.tensor(lens, dtype=torch.int32, device="cuda")
    out, lse = run(snapkv, q, pool, table, dl, max(lens) + room)
    check(q, pool, kind, table, lens, out, lse)
    again, _ = run(snapkv, q, pool, table, dl, max(lens) + room, lse=False)
    assert torch.equal(out, again)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dist", ["sharp", "flat", "far"])
def test_distributions(snapkv, dist, dtype):
    gen, lens = seeded(41), [1500, 40]
    q = rows(gen, 2, 8, 128, DT[dtype], "tokens")
    pool, table = mx_pool(gen, lens, 16, 2, 128, "fp8")
    if dist == "sharp":
        q.mul_(12)
    elif dist == "flat":
        q.zero_()
    else:                                                           # parts of the cache whose logits are far from the others'
        pool[1][table[0, :20].long()] += 3
        pool[1][table[0, 60:80].long()] -= 60
    out, lse = run(snapkv, q, pool, table, torch.tensor(lens, dtype=torch.int32, device="cuda"), 1500)
    check(q, pool, "fp8", table, lens, out, lse)


def test_small_and_large_scales_and_nan(snapkv):
    """Values at the ends of the scales' range, fp16 queries of 1e-4, and a block that reads as NaN, which only its own heads see."""
    gen, lens = seeded(42), [700, 300]
    q = rows(gen, 2, 4, 128, torch.float16, "tokens", scale=1e-4)
    pool, table = mx_pool(gen, lens, 16, 2, 128, "fp8")
    pool[1][table[0, 0].long()] = 10
    pool[3][table[0, 1].long()] = 10
    pool[3][table[1, :5].long()] = 127 + 9
    dl = torch.tensor(lens, dtype=torch.int32, device="cuda")
    out, lse = run(snapkv, q, pool, table, dl, 700)
    check(q, pool, "fp8", table, lens, out, lse)
    pool[3][table[1, 3].long(), 5, 1, 2] = 255                      # values of KV head 1, elements 64 .. 95
    pool[1][table[0, 3].long(), 5, 0, 0] = 255                      # a key of KV head 0
    bad, bad_lse = run(snapkv, q, pool, table, dl, 700)
    torch.cuda.synchronize()
    assert bad[0, :2].isnan().all() and bad_lse[0, :2].isnan().all() and torch.equal(bad[0, 2:], out[0, 2:])
    assert torch.equal(bad[1, :2], out[1, :2]) and bad[1, 2:, 64:96].isnan().all() and torch.equal(bad_lse[1], lse[1])
    assert torch.equal(bad[1, 2:, :64], out[1, 2:, :64]) and torch.equal(bad[1, 2:, 96:], out[1, 2:, 96:])


def test_queries_of_nan_and_infinity(snapkv):
    gen, lens = seeded(43), [900, 0]
    q = rows(gen, 2, 4, 64, torch.bfloat16, "tokens")
    pool, table = mx_pool(gen, lens, 16, 2, 64, "fp4")
    dl = torch.tensor(lens, dtype=torch.int32, device="cuda")
    want = run(snapkv, q, pool, table, dl, 900)
    q[0, 1, 3] = float("nan")
    got = run(snapkv, q, pool, table, dl, 900)
    torch.cuda.synchronize()
    assert got[0][0, 1].isnan().all() and bool(got[1][0, 1].isnan())
    keep = [0, 2, 3]
    assert torch.equal(got[0][0, keep], want[0][0, keep]) and torch.equal(got[1][0, keep], want[1][0, keep])
    assert (got[0][1] == 0).all() and (got[1][1] == -float("inf")).all()


def test_lengths_and_table_entries_are_clamped(snapkv):
    gen = seeded(44)
    q = rows(gen, 3, 4, 64, torch.bfloat16, "tokens")
    pool, table = mx_pool(gen, [100, 100, 100], 16, 2, 64, "fp8", spare=0)
    for s in (pool[1], pool[3]):
        s[s == 255] = 120
    table[2, 1], table[2, 2] = -3, 1 << 30
    lens = torch.tensor([-5, 1 << 30, 60], dtype=torch.int32, device="cuda")
    out, lse = run(snapkv, q, pool, table, lens, 100)
    check(q, pool, "fp8", table, [0, 100, 60], out, lse)


def test_step_equals_the_step_over_the_rows_read_back(snapkv):
    gen, B, S, page = seeded(45), 3, 1300, 16
    q = rows(gen, B, 16, 128, torch.bfloat16, "tokens")
    pool, table = mx_pool(gen, [S] * B, page, 4, 128, "fp4")
    k, v = (torch.empty((B * S, 4, 128), device="cuda", dtype=torch.bfloat16) for _ in range(2))
    cu, zero = torch.arange(0, (B + 1) * S, S, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
    snapkv.snapkv_read_paged_mx(*pool, table, zero, k, v, cu_seqlens=cu)
    kp, vp = (torch.zeros((pool[0].shape[0], page, 4, 128), device="cuda", dtype=torch.bfloat16) for _ in range(2))
    snapkv.snapkv_append_paged(k, v, kp, vp, table, zero, cu_seqlens=cu)
    dl = torch.full((B,), S, dtype=torch.int32, device="cuda")
    out, lse = run(snapkv, q, pool, table, dl, S)
    want, want_lse = torch.empty_like(out), torch.empty_like(lse)
    snapkv.snapkv_decode_attention_paged(q, kp, vp, table, dl, S, want, want_lse)
    torch.cuda.synchronize()
    assert (lse - want_lse).abs().max() <= 1e-4
    assert ((out.double() - want.double()).abs() <= 2.0 ** -7 * want.abs() + 2.0 ** -12 * float(v.abs().max())).all()


def test_pool_beyond_32_bit_offsets(snapkv):
    page, Hkv, D = 128, 16, 128
    pages = (1 << 32) // (page * Hkv * D) + 30
    pool = [torch.empty((pages, page, Hkv, n), device="cuda", dtype=torch.uint8) for n in (D, D // 32, D, D // 32)]
    small, order = mx_pool(seeded(46), [380], page, Hkv, D, "fp8", spare=0)
    table = torch.tensor([[pages - 1, 3, pages - 20]], dtype=torch.int32, device="cuda")
    for big, part in zip(pool, small):
        big[table[0].long()] = part[order[0, :3].long()]
    q = rows(seeded(47), 1, 16, D, torch.bfloat16, "tokens")
    out, lse = run(snapkv, q, pool, table, torch.tensor([380], dtype=torch.int32, device="cuda"), 384)
    check(q, small, "fp8", order, [380], out, lse)


def test_workspaces_hold_nothing_between_calls(snapkv):
    """A workspace full of NaN, and captured steps of two shapes that share one, replayed with other lengths."""
    gen, sets = seeded(48), []
    for lens, Hq, Hkv, kind in (([3000, 100], 16, 4, "fp8"), ([5000], 8, 8, "fp4")):
        pool, table = mx_pool(gen, lens, 16, Hkv, 128, kind)
        sets.append([rows(gen, len(lens), Hq, 128, torch.bfloat16, "tokens"), pool, table, torch.tensor(lens, dtype=torch.int32, device="cuda"), max(lens), kind])
    need = [snapkv.snapkv_decode_paged_mx_workspace_bytes(s[0].shape[0], s[0].shape[1], s[1][0].shape[2], 128, s[4]) for s in sets]
    assert min(need) > 0
    ws = torch.full((max(need),), 255, dtype=torch.uint8, device="cuda")
    for s in sets:
        want = run(snapkv, *s[:5])
        ws.fill_(255)
        got = run(snapkv, *s[:5], workspace=ws)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    graphs, outs = [], []
    torch.cuda.synchronize()
    for s in sets:
        o = (torch.empty_like(s[0]), torch.empty(s[0].shape[:2], device="cuda"))
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            snapkv.snapkv_decode_attention_paged_mx(s[0], *s[1], s[2], s[3], s[4], *o, workspace=ws)
        outs.append(o)
    for rep in range(4):
        for s, l in zip(sets, [[3000 - 7 * rep, 1 + rep], [5000 - 1111 * rep]]):
            s[0].normal_(generator=gen)
            s[3].copy_(torch.tensor(l))
        want = [run(snapkv, *s[:5]) for s in sets]
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            assert torch.equal(o[0], w[0]) and torch.equal(o[1], w[1])


def test_steps_on_two_streams_with_their_own_workspaces(snapkv):
    gen, sets, want = seeded(49), [], []
    for _ in range(2):
        pool, table = mx_pool(gen, [4000], 16, 4, 64, "fp8")
        s = (rows(gen, 1, 8, 64, torch.float16, "tokens"), pool, table, torch.tensor([4000], dtype=torch.int32, device="cuda"), 4000)
        sets.append((s, torch.empty(snapkv.snapkv_decode_paged_mx_workspace_bytes(1, 8, 4, 64, 4000), dtype=torch.uint8, device="cuda")))
        want.append(run(snapkv, *s))
    streams = [torch.cuda.Stream() for _ in sets]
    outs = [[(torch.empty((1, 8, 64), device="cuda", dtype=torch.float16), torch.empty((1, 8), device="cuda")) for _ in range(10)] for _ in sets]
    torch.cuda.synchronize()
    for i in range(10):
        for (s, ws), st, o in zip(sets, streams, outs):
            snapkv.snapkv_decode_attention_paged_mx(s[0], *s[1], *s[2:], *o[i], workspace=ws, stream=st)
    torch.cuda.synchronize()
    for w, o in zip(want, outs):
        assert all(torch.equal(a, w[0]) and torch.equal(b, w[1]) for a, b in o)
    with pytest.raises(ValueError, match="workspace"):
        s = sets[0][0]
        snapkv.snapkv_decode_attention_paged_mx(s[0], *s[1], *s[2:], *outs[0][0], stream=streams[0])
