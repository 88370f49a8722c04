"""snapkv_append_paged_mx and snapkv_read_paged_mx against the fp64 oracle: codes and scale bytes exactly."""
import numpy as np
import pytest
import torch

from oracle import mx_oracle as orc
from oracle import serve_oracle
from serve_checks import DT, W24, half_step, num, offsets, rows, seeded, tables

pytestmark = pytest.mark.gpu


def empty_pool(pages, page, Hkv, D, kind, fill=0x5A):
    width = D if kind == "fp8" else D // 2
    make = lambda n: torch.full((pages, page, Hkv, n), fill, device="cuda", dtype=torch.uint8)
    return [make(width), make(D // 32), make(width), make(D // 32)]


def expected(pool, kind, k, v, table, starts, cu):
    """The four parts of the pool after rows k, v (float64, rotated) went in."""
    parts = [t.cpu().numpy().copy() for t in pool]
    pages, page = parts[0].shape[:2]
    for b in range(len(starts)):
        for t in range(int(cu[b]), int(cu[b + 1])):
            r = int(starts[b]) + t - int(cu[b])
            if r < 0 or r // page >= table.shape[1] or not 0 <= table[b, r // page] < pages:
                continue
            at = (table[b, r // page], r % page)
            for i, x in ((0, k), (2, v)):
                codes, scales = orc.quantise(x[t], kind)
                parts[i][at], parts[i + 1][at] = orc.pack(codes, kind), scales
    return parts


CASES = [   # lengths, starts, page, Hq, Hkv, D, rot, interleaved, dtype, layout
    ([1], [0], 16, 4, 2, 128, 128, False, "bf16", "tokens"),
    ([1, 1, 1], [5, 0, 40], 16, 32, 8, 128, 128, False, "bf16", "fused"),
    ([33, 0, 7, 1], [0, 3, 30, 15], 16, 8, 2, 128, 128, True, "f16", "heads"),
    ([40, 21], [0, 9], 7, 6, 3, 64, 64, False, "bf16", "tokens"),
    ([40, 21], [1, 9], 1, 2, 1, 64, 32, False, "f16", "fused"),
    ([19, 5], [0, 100], 24, 4, 4, 128, 64, False, "f32", "heads"),
    ([19, 5], [2, 100], 128, 4, 4, 64, 64, True, "f32", "tokens"),
    ([19, 65], [2, 100], 8, 5, 5, 128, 0, False, "bf16", "heads"),
    ([30], [2], 16, 3, 3, 64, 16, True, "bf16", "tokens"),
    ([30], [2], 16, 3, 1, 128, 16, False, "f16", "tokens"),
    ([30], [2], 16, 3, 1, 128, 8, False, "f32", "tokens"),
    ([30, 4], [2, 0], 16, 3, 1, 128, 112, False, "bf16", "heads"),
    ([600, 523], [0, 77], 32, 2, 2, 64, 64, False, "bf16", "tokens"),
]


@pytest.mark.parametrize("kind", ["fp8", "fp4"])
@pytest.mark.parametrize("n", range(len(CASES)))
def test_append_and_read(snapkv, n, kind):
    lengths, starts, page, Hq, Hkv, D, rot, inter, dt, layout = CASES[n]
    gen, dtype, B, T = seeded(900 + n), DT[dt], len(lengths), sum(lengths)
    q, k, v = (rows(gen, T, h, D, dtype, layout, scale=s) for h, s in ((Hq, 1.0), (Hkv, 3.0), (Hkv, 1.0)))
    k.mul_(torch.exp(2 * torch.randn((Hkv, D), generator=gen, device="cuda")).to(dtype))
    need = [-(-(a + m) // page) for a, m in zip(starts, lengths)]
    pool = empty_pool(sum(need) + 2, page, Hkv, D, kind)
    table = torch.full((B, max(need) + 1), -1, dtype=torch.int32, device="cuda")
    order = torch.randperm(sum(need) + 2, generator=gen, device="cuda").to(torch.int32)
    for b in range(B):
        table[b, :need[b]] = order[sum(need[:b]):sum(need[:b + 1])]
    cu, ds = offsets(lengths), torch.tensor(starts, dtype=torch.int32, device="cuda")
    kw, turned_k, turned_q = dict(cu_seqlens=cu), num(k), num(q)
    if rot:
        positions = torch.cat([torch.arange(3 * a, 3 * a + m) for a, m in zip(starts, lengths)]).to(torch.int32).cuda()
        cos, sin = tables(700 + max(starts) * 3, rot // 2)
        q_out, k_out = torch.full((T, Hq, D), 7.0, device="cuda", dtype=dtype), torch.full((T, Hkv, D), 7.0, device="cuda", dtype=dtype)
        kw.update(positions=positions, cos=cos, sin=sin, interleaved=inter, q=q, q_out=q_out, k_out=k_out)
        turned_k, turned_q = (serve_oracle.rotate(num(x), positions.tolist(), num(cos), num(sin), inter) for x in (k, q))
    want = expected(pool, kind, turned_k, num(v), table.cpu().numpy(), starts, cu.tolist())
    snapkv.snapkv_append_paged_mx(k, v, *pool, table, ds, **kw)
    torch.cuda.synchronize()
    for got, w in zip(pool, want):
        assert np.array_equal(got.cpu().numpy(), w)
    if rot:
        for got, w, x in ((q_out, turned_q, q), (k_out, turned_k, k)):
            reach = 2 * num(x).__abs__().max(axis=-1, keepdims=True)
            assert (np.abs(num(got) - w) <= half_step(dtype) * np.abs(w) + 4 * W24 * reach).all()
    # back, to token-major and head-major storage, in every type
    seen = [orc.values(orc.unpack(want[i], kind), want[i + 1], kind) for i in (0, 2)]
    for dt_out in ("bf16", "f16", "f32"):
        for lay in ("tokens", "heads"):
            ko, vo = (rows(gen, T, Hkv, D, DT[dt_out], lay) for _ in range(2))
            snapkv.snapkv_read_paged_mx(*pool, table, ds, ko, vo, cu_seqlens=cu)
            torch.cuda.synchronize()
            for out, x in ((ko, seen[0]), (vo, seen[1])):
                for b in range(B):
                    r = starts[b] + np.arange(lengths[b])
                    w = x[table[b].cpu().numpy()[r // page], r % page]
                    exact = torch.from_numpy(w).to(DT[dt_out])     # (to_float64 -> type: one rounding, to nearest even)
                    assert torch.equal(out[cu[b]:cu[b + 1]].cpu(), exact)


@pytest.mark.parametrize("kind", ["fp8", "fp4"])
def test_every_code_is_reached_and_kept(snapkv, kind):
    """Values on the grid, halfway between and next to it, at the smallest and largest scales, and blocks with infinities and NaN."""
    grid, D = orc.GRID[kind], 128
    mids = (grid[1:] + grid[:-1]) / 2
    vals = np.concatenate([grid, mids, np.nextafter(mids.astype(np.float32), np.float32(0)), np.nextafter(mids.astype(np.float32), np.float32(1e9))])
    vals = np.concatenate([vals, -vals])
    vals = np.pad(vals, (0, -len(vals) % 31)).reshape(-1, 31)
    top = np.full((len(vals), 1), grid[-1])
    blocks = np.concatenate([top, vals], axis=1).astype(np.float32)
    rows_ = []
    for e in (0, -3, 60, 119, -117, -126, -140):
        x = np.ldexp(blocks.astype(np.float64), e)
        rows_.append(np.where(np.abs(x) > 3.4e38, 1.0, x).astype(np.float32))
    for bad in (np.inf, -np.inf, np.nan):
        x = blocks[:2].copy()
        x[0, 7] = bad
        rows_.append(x)
    x = np.concatenate(rows_)
    x = np.concatenate([x, np.zeros((-len(x) % 4, 32), np.float32)]).reshape(-1, 1, D)
    T = len(x)
    k = torch.from_numpy(x).cuda()
    pool = empty_pool(T, 1, 1, D, kind)
    table = torch.arange(T, dtype=torch.int32, device="cuda").view(1, T)
    zero, cu = torch.zeros(1, dtype=torch.int32, device="cuda"), offsets([T])
    snapkv.snapkv_append_paged_mx(k, -k, *pool, table, zero, cu_seqlens=cu)
    ko, vo = torch.empty_like(k), torch.empty_like(k)
    snapkv.snapkv_read_paged_mx(*pool, table, zero, ko, vo, cu_seqlens=cu)
    torch.cuda.synchronize()
    for i, s, out in ((0, 1.0, ko), (2, -1.0, vo)):
        codes, scales = orc.quantise(s * x.astype(np.float64), kind)
        assert np.array_equal(pool[i].cpu().numpy()[:, 0], orc.pack(codes, kind)) and np.array_equal(pool[i + 1].cpu().numpy()[:, 0], scales)
        assert np.array_equal(num(out), orc.values(codes, scales, kind).astype(np.float32).astype(np.float64), equal_nan=True)
    if kind == "fp8":
        assert len(np.unique(pool[0].cpu().numpy())) == 254          # all but the two NaN


@pytest.mark.parametrize("kind", ["fp8", "fp4"])
def test_codes_of_pages_that_others_wrote(snapkv, kind):
    """All codes under scales from 2^-117 to 2^119, the codes that are NaN, and the scale that is."""
    D, n = 64, 256 if kind == "fp8" else 256
    codes = torch.arange(256, dtype=torch.uint8, device="cuda").repeat(1 if kind == "fp8" else 1)
    width = D if kind == "fp8" else D // 2
    scales = [10, 11, 100, 127, 140, 246, 255]
    pages = len(scales)
    kp = codes.view(1, 256 // width, 1, width).repeat(pages, 1, 1, 1).contiguous()
    ks = torch.tensor(scales, dtype=torch.uint8, device="cuda").view(-1, 1, 1, 1).repeat(1, 256 // width, 1, D // 32).contiguous()
    T = pages * (256 // width)
    table = torch.arange(pages, dtype=torch.int32, device="cuda").view(1, -1)
    for dtype in DT.values():
        out = torch.empty((2, T, 1, D), device="cuda", dtype=dtype)
        snapkv.snapkv_read_paged_mx(kp, ks, kp, ks, table, torch.zeros(1, dtype=torch.int32, device="cuda"), out[0], out[1], cu_seqlens=offsets([T]))
        torch.cuda.synchronize()
        want = orc.values(orc.unpack(kp.cpu().numpy(), kind), ks.cpu().numpy(), kind).reshape(T, 1, D)
        want = torch.from_numpy(want).to(dtype)
        assert torch.equal(out[0].cpu().nan_to_num(123.0, posinf=1e30, neginf=-1e30) if dtype != torch.float16 else out[0].cpu().nan_to_num(123.0, 999.0, -999.0),
                           want.nan_to_num(123.0, posinf=1e30, neginf=-1e30) if dtype != torch.float16 else want.nan_to_num(123.0, 999.0, -999.0))
        assert torch.equal(out[0].isnan(), out[1].isnan())


def test_rows_without_a_place_are_left_alone(snapkv):
    """Tokens before the first sequence and behind the last, rows before the first and behind the last column, entries of no page."""
    gen, D, Hkv, page, T = seeded(31), 64, 2, 4, 30
    k, v = (rows(gen, T, Hkv, D, torch.bfloat16, "tokens") for _ in range(2))
    table = torch.tensor([[2, 99, 1], [0, 3, -1]], dtype=torch.int32, device="cuda")
    starts = torch.tensor([-3, 5], dtype=torch.int32, device="cuda")
    cu = torch.tensor([2, 20, 27], dtype=torch.int32, device="cuda")
    pool = empty_pool(4, page, Hkv, D, "fp8")
    want = expected(pool, "fp8", num(k), num(v), table.cpu().numpy(), starts.tolist(), cu.tolist())
    snapkv.snapkv_append_paged_mx(k, v, *pool, table, starts, cu_seqlens=cu)
    torch.cuda.synchronize()
    for got, w in zip(pool, want):
        assert np.array_equal(got.cpu().numpy(), w)
    assert (want[0] == 0x5A).all(axis=-1).any()                      # (rows of pages that no token has)
    out = torch.full((2, T, Hkv, D), 77.0, device="cuda")
    snapkv.snapkv_read_paged_mx(*pool, table, starts, out[0], out[1], cu_seqlens=cu)
    torch.cuda.synchronize()
    for t in range(T):
        b = 0 if t < 20 else 1
        r = starts.tolist()[b] + t - cu.tolist()[b]
        has = 2 <= t < 27 and 0 <= r < 12 and 0 <= table.cpu()[b, max(r, 0) // page if 0 <= r < 12 else 0] < 4
        assert bool((out[0, t] == 77).all()) != has and bool((out[1, t] == 77).all()) != has


def test_pool_beyond_32_bit_offsets(snapkv):
    page, Hkv, D = 128, 16, 128
    pages = (1 << 32) // (page * Hkv * D) + 30
    pool = [torch.empty((pages, page, Hkv, n), device="cuda", dtype=torch.uint8) for n in (D, D // 32, D, D // 32)]
    gen, T = seeded(32), 200
    k, v = (rows(gen, T, Hkv, D, torch.float16, "tokens") for _ in range(2))
    table = torch.tensor([[pages - 1, 3]], dtype=torch.int32, device="cuda")
    zero, cu = torch.zeros(1, dtype=torch.int32, device="cuda"), offsets([T])
    snapkv.snapkv_append_paged_mx(k, v, *pool, table, zero, cu_seqlens=cu)
    ko, vo = torch.empty_like(k), torch.empty_like(v)
    snapkv.snapkv_read_paged_mx(*pool, table, zero, ko, vo, cu_seqlens=cu)
    torch.cuda.synchronize()
    for x, out in ((k, ko), (v, vo)):
        codes, scales = orc.quantise(num(x), "fp8")
        assert np.array_equal(num(out), orc.values(codes, scales, "fp8"))


def test_captured_appends_and_reads(snapkv):
    """One graph of both calls, replayed with new rows, and the eager calls between."""
    gen, D, Hkv, page, B = seeded(33), 128, 4, 16, 5
    q, k, v = (rows(gen, B, h, D, torch.bfloat16, "tokens") for h in (8, Hkv, Hkv))
    pool = empty_pool(12, page, Hkv, D, "fp4")
    table = torch.randperm(12, generator=gen, device="cuda")[:10].to(torch.int32).view(B, 2)
    starts = torch.arange(B, dtype=torch.int32, device="cuda") * 3
    cos, sin = tables(64, 64)
    qo, ko, vo = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)

    def both():
        snapkv.snapkv_append_paged_mx(k, v, *pool, table, starts, cos=cos, sin=sin, q=q, q_out=qo)
        snapkv.snapkv_read_paged_mx(*pool, table, starts, ko, vo)

    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for rep in range(4):
        for t in (q, k, v):
            t.normal_(generator=gen)
        starts.add_(1)
        both()
        want = [t.clone() for t in (qo, ko, vo, *pool)]
        for t in (qo, ko, vo):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((qo, ko, vo, *pool), want))
