"""snapkv_decode_attention_paged against the fp64 oracle; bounds in serve_checks.py."""
import numpy as np
import pytest
import torch

from oracle import serve_oracle as orc
from serve_checks import DT, check_attention, fill_rows, num, pool, rows, seeded

pytestmark = pytest.mark.gpu


def run(snapkv, q, kp, vp, table, lens, max_len, lse=True, workspace=None, stream=None):
    out = torch.full(q.shape, 77.0, device="cuda", dtype=q.dtype)
    out_lse = torch.full(q.shape[:2], 77.0, device="cuda") if lse else None
    snapkv.snapkv_decode_attention_paged(q, kp, vp, table, lens, max_len, out, out_lse, workspace=workspace, stream=stream)
    return out, out_lse


def check(q, kp, vp, table, lens, out, lse):
    torch.cuda.synchronize()
    zero = lambda t: np.nan_to_num(num(t))                    # (rows of nobody hold NaN)
    want, want_lse, spread, reach = orc.decode_paged(num(q), zero(kp), zero(vp), table.cpu().numpy(), lens)
    some = np.array(lens) > 0
    got = num(out)
    assert (got[~some] == 0).all()
    if lse is not None:
        assert np.isneginf(num(lse)[~some]).all()
    if some.any():
        check_attention(got[some], num(lse)[some] if lse is not None else None, want[some], want_lse[some], spread[some], reach[some],
                        max(lens), q.dtype, parts=True)


CASES = [   # lens, page, Hq, Hkv, D, dtype, room beyond the longest
    ([1], 16, 4, 4, 128, "bf16", 0),
    ([0, 1, 15, 16, 17, 31, 32, 33], 16, 8, 2, 64, "bf16", 5),
    ([127, 128, 129, 255, 256, 257], 8, 16, 1, 128, "f16", 0),
    ([511, 512, 513, 1], 32, 32, 8, 128, "bf16", 0),
    ([2113], 16, 32, 8, 128, "bf16", 400),
    ([4097, 3], 24, 3, 3, 64, "f16", 0),
    ([1000, 7, 0, 2500], 1, 6, 2, 128, "bf16", 0),
    ([300, 301], 7, 10, 5, 64, "bf16", 1),
    ([777], 1024, 4, 1, 128, "f16", 0),
    ([20000], 64, 4, 2, 64, "bf16", 0),
    ([900, 1], 128, 24, 24, 128, "bf16", 31000),              # cut for far longer sequences
    ([64] * 150, 16, 2, 2, 64, "f16", 0),
    ([5000, 1, 777, 0, 4096, 130, 129], 16, 8, 4, 128, "bf16", 0),
    ([1700] * 9 + [40, 3], 8, 3, 3, 64, "bf16", 300),
    ([2113], 16, 8, 2, 64, "f16", 129000),                    # shares as long as the sequence asks for, not the cache
    ([5000, 300, 129, 2], 32, 8, 8, 128, "bf16", 60000),
    ([3000] + [1] * 40, 16, 4, 2, 64, "bf16", 20000),
]


@pytest.mark.parametrize("n", range(len(CASES)))
def test_step_matches_oracle(snapkv, n):
    lens, page, Hq, Hkv, D, dt, room = CASES[n]
    gen, dtype = seeded(200 + n), DT[dt]
    q = rows(gen, len(lens), Hq, D, dtype, "tokens")
    kp, vp, table = pool(gen, [x + room for x in lens], page, Hkv, D, dtype)
    fill_rows(gen, kp, vp, table, lens)
    dl = torch.tensor(lens, dtype=torch.int32, device="cuda")
    most = max(lens) + room
    out, lse = run(snapkv, q, kp, vp, table, dl, most)
    check(q, kp, vp, table, lens, out, lse)
    again, _ = run(snapkv, q, kp, vp, table, dl, most, lse=False)
    assert torch.equal(out, again)


@pytest.mark.parametrize("kind", ["sharp", "flat", "far"])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_distributions(snapkv, kind, dtype):
    """One row takes all, all alike, and logits that differ so much between parts of the cache that whole parts vanish."""
    gen, lens = seeded(3), [1500, 40]
    q = rows(gen, 2, 8, 128, DT[dtype], "tokens")
    kp, vp, table = pool(gen, lens, 16, 2, 128, DT[dtype])
    fill_rows(gen, kp, vp, table, lens)
    if kind == "sharp":
        q.mul_(12)
    elif kind == "flat":
        q.zero_()
    else:
        q.copy_(q.abs() + 1)
        kp[table[0, :20].long()] -= 4
        kp[table[0, 60:80].long()] += 4
    out, lse = run(snapkv, q, kp, vp, table, torch.tensor(lens, dtype=torch.int32, device="cuda"), 1500)
    check(q, kp, vp, table, lens, out, lse)


def test_lengths_and_table_entries_are_clamped(snapkv):
    gen = seeded(4)
    q = rows(gen, 3, 4, 64, torch.bfloat16, "tokens")
    kp, vp, table = pool(gen, [100, 100, 100], 16, 2, 64, torch.bfloat16, fill=0.5)
    fill_rows(gen, kp, vp, table, [100] * 3)
    table[2, 1], table[2, 2] = -3, 1 << 30
    lens = torch.tensor([-5, 1 << 30, 60], dtype=torch.int32, device="cuda")
    out, lse = run(snapkv, q, kp, vp, table, lens, 100)
    check(q, kp, vp, table, [0, 100, 60], out, lse)


def test_step_equals_the_step_over_a_contiguous_cache(snapkv):
    """The same rows in both kinds of cache: equal up to the last rounding."""
    gen, B, S = seeded(5), 3, 1300
    q = rows(gen, B, 16, 128, torch.bfloat16, "tokens")
    k, v = (torch.randn((B, 4, S, 128), generator=gen, device="cuda").bfloat16() for _ in range(2))
    kp, vp, table = pool(gen, [S] * B, 16, 4, 128, torch.bfloat16)
    snapkv.snapkv_append_paged(k.permute(0, 2, 1, 3).reshape(B * S, 4, 128), v.permute(0, 2, 1, 3).reshape(B * S, 4, 128), kp, vp, table,
                               torch.zeros(B, dtype=torch.int32, device="cuda"),
                               cu_seqlens=torch.arange(0, (B + 1) * S, S, dtype=torch.int32, device="cuda"))
    out, lse = run(snapkv, q, kp, vp, table, torch.full((B,), S, dtype=torch.int32, device="cuda"), S)
    want, want_lse = torch.empty((B, 16, 128), device="cuda"), torch.empty((B, 16), device="cuda")
    snapkv.snapkv_decode_attention(q, k, v, S, want, want_lse)
    torch.cuda.synchronize()
    assert (out.double() - want.double()).abs().max() <= 2.0 ** -8 * want.abs().max() + 2e-4 * float(v.float().abs().max())
    assert (lse - want_lse).abs().max() <= 2e-4


def test_pool_beyond_32_bit_offsets(snapkv):
    page, Hkv, D = 128, 8, 128
    pages = (1 << 31) // (page * Hkv * D) + 40
    kp = torch.empty((pages, page, Hkv, D), device="cuda", dtype=torch.bfloat16)
    vp = torch.empty_like(kp)
    table = torch.tensor([[pages - 1, 3, pages - 20]], dtype=torch.int32, device="cuda")
    gen = seeded(6)
    for p in table[0].tolist():
        for t in (kp, vp):
            t[p] = torch.randn((page, Hkv, D), generator=gen, device="cuda").bfloat16()
    q = rows(gen, 1, 16, D, torch.bfloat16, "tokens")
    out, lse = run(snapkv, q, kp, vp, table, torch.tensor([380], dtype=torch.int32, device="cuda"), 384)
    at = table[0].long()
    small = torch.tensor([[0, 1, 2]], dtype=torch.int32, device="cuda")
    check(q, kp[at], vp[at], small, [380], out, lse)


def test_workspaces_hold_nothing_between_calls(snapkv):
    """A workspace full of NaN, one that another shape has used, and two captured steps that share one."""
    gen = seeded(7)
    sets = []
    for lens, Hq, Hkv in (([3000, 100], 16, 4), ([5000], 8, 8)):
        kp, vp, table = pool(gen, lens, 16, Hkv, 128, torch.bfloat16)
        fill_rows(gen, kp, vp, table, lens)
        sets.append((rows(gen, len(lens), Hq, 128, torch.bfloat16, "tokens"), kp, vp, table, torch.tensor(lens, dtype=torch.int32, device="cuda"), max(lens)))
    need = [snapkv.snapkv_decode_paged_workspace_bytes(s[0].shape[0], s[0].shape[1], s[1].shape[2], 128, s[5]) for s in sets]
    assert min(need) > 0
    ws = torch.full((max(need),), 255, dtype=torch.uint8, device="cuda")
    want = [run(snapkv, *s) for s in sets]
    for s, w in zip(sets, want):
        ws.fill_(255)
        got = run(snapkv, *s, workspace=ws)
        assert torch.equal(got[0], w[0]) and torch.equal(got[1], w[1])
    graphs, outs = [], []
    torch.cuda.synchronize()
    for s in sets:
        o = (torch.empty_like(s[0]), torch.empty(s[0].shape[:2], device="cuda"))
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            snapkv.snapkv_decode_attention_paged(*s, *o, workspace=ws)
        outs.append(o)
    for rep in range(4):
        lens = [[3000 - 7 * rep, 1 + rep], [5000 - 1111 * rep]]
        for s, l in zip(sets, lens):
            s[0].normal_(generator=gen)
            s[4].copy_(torch.tensor(l))
        want = [run(snapkv, *s) for s in sets]
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            assert torch.equal(o[0], w[0]) and torch.equal(o[1], w[1])
        check(sets[0][0], *sets[0][1:4], lens[0], *outs[0])


def test_steps_on_two_streams_with_their_own_workspaces(snapkv):
    gen, sets, want = seeded(8), [], []
    for _ in range(2):
        kp, vp, table = pool(gen, [4000], 16, 4, 64, torch.float16)
        fill_rows(gen, kp, vp, table, [4000])
        s = (rows(gen, 1, 8, 64, torch.float16, "tokens"), kp, vp, table, torch.tensor([4000], dtype=torch.int32, device="cuda"), 4000)
        sets.append((s, torch.empty(snapkv.snapkv_decode_paged_workspace_bytes(1, 8, 4, 64, 4000), dtype=torch.uint8, device="cuda")))
        want.append(run(snapkv, *s))
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    outs = [[(torch.empty_like(s[0]), torch.empty((1, 8), device="cuda")) for _ in range(10)] for s, _ in sets]
    torch.cuda.synchronize()
    for i in range(10):
        for (s, ws), st, o in zip(sets, streams, outs):
            snapkv.snapkv_decode_attention_paged(*s, *o[i], workspace=ws, stream=st)
    torch.cuda.synchronize()
    for w, o in zip(want, outs):
        assert all(torch.equal(a, w[0]) and torch.equal(b, w[1]) for a, b in o)
    with pytest.raises(ValueError, match="workspace"):
        snapkv.snapkv_decode_attention_paged(*sets[0][0], *outs[0][0], stream=streams[0])
