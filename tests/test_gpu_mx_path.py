"""The steps over microscaled pages and shared prefixes run together, as a serving program runs them: prompts go into a cache of 8 or 4 bits and
through attention, leave it to be compressed, the kept rows go into pages of their own, and several answers to each prompt are
generated over one copy of them (the steps captured once).  Every stage is checked on what the stage before it stored."""
import numpy as np
import pytest
import torch

from mx_checks import check_step, mx_values
from oracle import mx_oracle as orc
from oracle import serve_oracle
from serve_checks import check_attention, half_step, num, offsets, seeded, tables
from test_gpu_mx_cache import empty_pool, expected

pytestmark = pytest.mark.gpu

LENGTHS, Hq, Hkv, D, W, P, C, PAGE, ANSWERS, STEPS = [700, 300, 1103], 8, 2, 128, 32, 7, 256, 16, [3, 1, 5], 4


@pytest.mark.parametrize("kind", ["fp8", "fp4"])
def test_prompts_to_generated_answers(snapkv, kind):
    gen, dtype, B, T = seeded(61), torch.bfloat16, len(LENGTHS), sum(LENGTHS)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    cos, sin = tables(2048, D // 2)
    q, k, v = (t.view(T, -1, D) for t in torch.randn((T, (Hq + 2 * Hkv) * D), generator=gen, device="cuda").to(dtype).split([Hq * D, Hkv * D, Hkv * D], dim=1))
    cu = offsets(LENGTHS)
    at = cu.tolist()

    def pages_for(lens):
        need = [-(-n // PAGE) for n in lens]
        order = torch.randperm(sum(need) + 2, generator=gen, device="cuda").to(torch.int32)
        table = torch.zeros((len(lens), max(need)), dtype=torch.int32, device="cuda")
        for b, n in enumerate(need):
            table[b, :n] = order[sum(need[:b]):sum(need[:b + 1])]
        return empty_pool(sum(need) + 2, PAGE, Hkv, D, kind), table

    # the prompts into pages, their rotated keys once more for the attention over them
    pool, table = pages_for(LENGTHS)
    qt, kt = torch.empty((T, Hq, D), device="cuda", dtype=dtype), torch.empty((T, Hkv, D), device="cuda", dtype=dtype)
    snapkv.snapkv_append_paged_mx(k, v, *pool, table, i32([0] * B), cu_seqlens=cu, cos=cos, sin=sin, q=q, q_out=qt, k_out=kt)
    positions = [p for n in LENGTHS for p in range(n)]
    turned = serve_oracle.rotate(num(k), positions, num(cos), num(sin), False)
    empty = empty_pool(pool[0].shape[0], PAGE, Hkv, D, kind)
    torch.cuda.synchronize()
    for got, want in zip(pool, expected(empty, kind, turned, num(v), table.cpu().numpy(), [0] * B, at)):
        assert np.array_equal(got.cpu().numpy(), want)
    assert (np.abs(num(kt) - turned) <= half_step(dtype) * np.abs(turned) + 1e-5).all()
    out, lse = torch.empty((T, Hq, D), device="cuda", dtype=dtype), torch.empty((Hq, T), device="cuda")
    snapkv.snapkv_prompt_attention(qt, kt, v, cu, out, lse)
    torch.cuda.synchronize()
    want, want_lse, spread, reach = serve_oracle.prompt_attention(num(qt), num(kt), num(v), at)
    check_attention(num(out), num(lse).T, want, want_lse.T, spread, reach.T, max(LENGTHS), dtype, parts=False)

    # back out of the pages, head by head, and compressed
    kb, vb = (torch.empty((Hkv, T, D), device="cuda", dtype=dtype) for _ in range(2))
    snapkv.snapkv_read_paged_mx(*pool, table, i32([0] * B), kb.transpose(0, 1), vb.transpose(0, 1), cu_seqlens=cu)
    kept_k, kept_v, kept = [], [], []
    for b, L in enumerate(LENGTHS):
        a, e = at[b], at[b + 1]
        ok, ov = (torch.zeros((Hkv, C, D), device="cuda", dtype=dtype) for _ in range(2))
        oi = torch.zeros((Hkv, C), device="cuda", dtype=torch.int32)
        ks, vs = kb[:, a:e].contiguous(), vb[:, a:e].contiguous()
        n = snapkv.snapkv_compress(qt[e - W:e].transpose(0, 1).contiguous(), ks, vs, snapkv.POOL_MAX, P, C, ok, ov, oi)
        torch.cuda.synchronize()
        assert n == min(C, L)
        for h in range(Hkv):
            assert torch.equal(ok[h, :n], ks[h][oi[h, :n].long()]) and torch.equal(ov[h, :n], vs[h][oi[h, :n].long()])
        kept_k.append(ok[:, :n].transpose(0, 1))
        kept_v.append(ov[:, :n].transpose(0, 1))
        kept.append(n)

    # the kept rows into pages of their own: what was read from such pages goes back as it is; room for every answer's own rows
    N = sum(ANSWERS)
    cache, tables_ = pages_for(kept + [STEPS] * N)
    prefix_table, own_table = tables_[:B].contiguous(), tables_[B:, :1].contiguous()
    for b in range(B):
        snapkv.snapkv_append_paged_mx(kept_k[b], kept_v[b], *cache, prefix_table[b:b + 1], i32([0]), cu_seqlens=i32([0, kept[b]]))
        back = torch.empty((2, kept[b], Hkv, D), device="cuda", dtype=dtype)
        snapkv.snapkv_read_paged_mx(*cache, prefix_table[b:b + 1], i32([0]), back[0], back[1], cu_seqlens=i32([0, kept[b]]))
        torch.cuda.synchronize()
        assert torch.equal(back[0], kept_k[b]) and torch.equal(back[1], kept_v[b])

    # generated tokens: row t of each answer, position L + t; one step captured, replayed with the device's own counters
    groups = offsets(ANSWERS)
    lens, pos = i32([0] * N), i32([L for L, n in zip(LENGTHS, ANSWERS) for _ in range(n)])
    new = torch.randn((N, (Hq + 2 * Hkv) * D), generator=gen, device="cuda").to(dtype)
    qn, kn, vn = (t.view(N, -1, D) for t in new.split([Hq * D, Hkv * D, Hkv * D], dim=1))
    qr, o, l = torch.empty((N, Hq, D), device="cuda", dtype=dtype), torch.empty((N, Hq, D), device="cuda", dtype=dtype), torch.empty((N, Hq), device="cuda")
    prefix_lens = i32(kept)

    def step():
        snapkv.snapkv_append_paged_mx(kn, vn, *cache, own_table, lens, positions=pos, cos=cos, sin=sin, q=qn, q_out=qr)
        lens.add_(1)
        pos.add_(1)
        snapkv.snapkv_decode_attention_shared(qr, cache[0], cache[2], prefix_table, prefix_lens, max(kept), own_table, lens, STEPS, o, l,
                                              cu_groups=groups, k_scales=cache[1], v_scales=cache[3])

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    values = lambda: (mx_values(cache[0], cache[1], kind), mx_values(cache[2], cache[3], kind))
    spans = list(zip(groups.tolist()[:-1], groups.tolist()[1:]))
    for t in range(STEPS):
        new.copy_(torch.randn(new.shape, generator=gen, device="cuda"))
        if t == 2:
            step()                                               # (an eager step between the replays)
        else:
            graph.replay()
        torch.cuda.synchronize()
        assert lens.tolist() == [t + 1] * N
        for (s, scales), x in (((cache[0], cache[1]), serve_oracle.rotate(num(kn), [p - 1 for p in pos.tolist()], num(cos), num(sin), False)),
                               ((cache[2], cache[3]), num(vn))):
            codes, scale = orc.quantise(x, kind)
            page = own_table[:, 0].long()
            assert np.array_equal(s[page, t].cpu().numpy(), orc.pack(codes, kind)) and np.array_equal(scales[page, t].cpu().numpy(), scale)
        want = orc.decode_shared(num(qr), *values(), prefix_table.cpu().numpy(), kept, own_table.cpu().numpy(), [t + 1] * N, spans)
        check_step(o, l, *want, max(kept) + t + 1, dtype)
        # the same answers one by one, over a table that names the prompt's pages and then the answer's
        whole = torch.zeros((N, prefix_table.shape[1] + 1), dtype=torch.int32, device="cuda")
        full = [i for i, (n, m) in enumerate(zip(kept, ANSWERS)) for _ in range(m)]
        for i, b in enumerate(full):
            assert kept[b] % PAGE == 0 or kept[b] < C
            whole[i, :-(-kept[b] // PAGE)] = prefix_table[b, :-(-kept[b] // PAGE)]
            whole[i, kept[b] // PAGE] = own_table[i, 0] if kept[b] % PAGE == 0 else whole[i, kept[b] // PAGE]
        some = [i for i, b in enumerate(full) if kept[b] % PAGE == 0]
        o2, l2 = torch.empty((len(some), Hq, D), device="cuda", dtype=dtype), torch.empty((len(some), Hq), device="cuda")
        snapkv.snapkv_decode_attention_paged_mx(qr[some].contiguous(), *cache, whole[some].contiguous(), i32([kept[full[i]] + t + 1 for i in some]), max(kept) + STEPS, o2, l2)
        torch.cuda.synchronize()
        assert (l2 - l[some]).abs().max() <= 1e-4
        assert ((o2.double() - o[some].double()).abs() <= 2.0 ** -7 * o2.abs() + 2.0 ** -10).all()
