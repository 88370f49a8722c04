"""The steps around a prompt's cache run together, as a serving program runs them: a batch of prompts goes into pages and
through attention, is compressed with the attention's log-sum-exp, the kept rows move into pages of their own, and tokens are
generated over them (the steps captured once).  Every stage is checked on what the stage before it stored; bounds in
serve_checks.py."""
import numpy as np
import pytest
import torch

from oracle import serve_oracle as orc
from serve_checks import check_attention, num, offsets, pool, seeded, tables

pytestmark = pytest.mark.gpu

LENGTHS, Hq, Hkv, D, W, P, C, PAGE, STEPS = [900, 300, 1503], 8, 2, 128, 32, 7, 512, 16, 5


def test_prompts_to_generated_tokens(snapkv):
    gen, dtype, B, T = seeded(1), torch.bfloat16, len(LENGTHS), sum(LENGTHS)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    cos, sin = tables(2048, D // 2)
    q, k, v = (t.view(T, -1, D) for t in torch.randn((T, (Hq + 2 * Hkv) * D), generator=gen, device="cuda").to(dtype).split(
        [Hq * D, Hkv * D, Hkv * D], dim=1))
    cu = offsets(LENGTHS)
    at = cu.tolist()

    # the prompts' rows go into pages, keys and queries turned
    kp, vp, table = pool(gen, LENGTHS, PAGE, Hkv, D, dtype)
    qt = torch.empty((T, Hq, D), device="cuda", dtype=dtype)
    kt = torch.empty((Hkv, T, D), device="cuda", dtype=dtype).transpose(0, 1)       # head by head, as the compression takes them
    snapkv.snapkv_append_paged(k, v, kp, vp, table, i32([0] * B), cu_seqlens=cu, cos=cos, sin=sin, q=q, q_out=qt, k_out=kt)

    out, lse = torch.empty((T, Hq, D), device="cuda", dtype=dtype), torch.empty((Hq, T), device="cuda")
    snapkv.snapkv_prompt_attention(qt, kt, v, cu, out, lse)
    torch.cuda.synchronize()
    want, want_lse, spread, reach = orc.prompt_attention(num(qt), num(kt), num(v), at)
    check_attention(num(out), num(lse).T, want, want_lse.T, spread, reach.T, max(LENGTHS), dtype, parts=False)

    # compressed with the window rows' log-sum-exp; from the pages the scores, and so the rows, are the same within rounding
    kept_k, kept_v, kept = [], [], []
    for b, L in enumerate(LENGTHS):
        a, e = at[b], at[b + 1]
        q_win = qt[e - W:e].transpose(0, 1).contiguous()
        kb, vb = kt[a:e].transpose(0, 1).contiguous(), v[a:e].transpose(0, 1).contiguous()
        ok, ov = (torch.zeros((Hkv, C, D), device="cuda", dtype=dtype) for _ in range(2))
        oi = torch.zeros((Hkv, C), device="cuda", dtype=torch.int32)
        n = snapkv.snapkv_compress_lse(q_win, kb, vb, lse[:, e - W:e].contiguous(), snapkv.POOL_MAX, P, C, ok, ov, oi)
        assert n == min(C, L)
        for h in range(Hkv):
            assert torch.equal(ok[h, :n], kb[h][oi[h, :n].long()]) and torch.equal(ov[h, :n], vb[h][oi[h, :n].long()])
        if L > C:
            by_lse, by_scan = (torch.empty((Hkv, L - W), device="cuda") for _ in range(2))
            snapkv.snapkv_pooled_scores_lse(q_win, kb, lse[:, e - W:e].contiguous(), snapkv.POOL_MAX, P, by_lse)
            snapkv.snapkv_pooled_scores(q_win, kb, snapkv.POOL_MAX, P, by_scan)
            assert ((by_lse - by_scan).abs() <= 1e-3 * by_scan).all()
            pk, pv, pi = torch.zeros_like(ok), torch.zeros_like(ov), torch.zeros_like(oi)
            snapkv.snapkv_compress_paged(q_win, kp, vp, table[b, :-(-L // PAGE)].contiguous(), L, snapkv.POOL_MAX, P, C, pk, pv, pi)
            torch.cuda.synchronize()
            for h in range(Hkv):
                assert torch.equal(pk[h], kb[h][pi[h].long()]) and torch.equal(pv[h], vb[h][pi[h].long()])
                assert np.isin(num(pi[h]), num(oi[h])).mean() > 0.99        # (scores as near as rounding may change places)
        kept_k.append(ok[:, :n].permute(1, 0, 2))
        kept_v.append(ov[:, :n].permute(1, 0, 2))
        kept.append(n)

    # the kept rows move into pages with room for what will be generated
    ck, cv, ctable = pool(gen, [n + STEPS for n in kept], PAGE, Hkv, D, dtype)
    for b in range(B):
        snapkv.snapkv_append_paged(kept_k[b], kept_v[b], ck, cv, ctable[b:b + 1], i32([0]), cu_seqlens=i32([0, kept[b]]))

    # generated tokens: row kept + t, position L + t; one step captured, replayed with the device's own counters
    qn, kn, vn = (torch.empty((B, h, D), device="cuda", dtype=dtype) for h in (Hq, Hkv, Hkv))
    qr, o, l = torch.empty_like(qn), torch.empty_like(qn), torch.empty((B, Hq), device="cuda")
    starts, pos, lens = i32(kept), i32(LENGTHS), i32([n + 1 for n in kept])
    most = max(kept) + STEPS
    ws = torch.empty(snapkv.snapkv_decode_paged_workspace_bytes(B, Hq, Hkv, D, most), dtype=torch.uint8, device="cuda")

    def step():
        snapkv.snapkv_append_paged(kn, vn, ck, cv, ctable, starts, positions=pos, cos=cos, sin=sin, q=qn, q_out=qr)
        snapkv.snapkv_decode_attention_paged(qr, ck, cv, ctable, lens, most, o, l, workspace=ws)
        for t in (starts, pos, lens):
            t.add_(1)

    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    for t in range(STEPS):
        for x in (qn, kn, vn):
            x.normal_(generator=gen)
        if t == 0:
            step()
        elif t == 1:
            with torch.cuda.graph(graph):
                step()
            graph.replay()
        else:
            graph.replay()
        torch.cuda.synchronize()
        cp, sp = num(cos), num(sin)
        turned = orc.rotate(num(kn), [L + t for L in LENGTHS], cp, sp, False)
        for b in range(B):
            r = kept[b] + t
            row = ck[int(ctable[b, r // PAGE]), r % PAGE]
            assert np.abs(num(row) - turned[b]).max() <= 2.0 ** -8 * np.abs(turned[b]).max() * 1.01
            assert torch.equal(cv[int(ctable[b, r // PAGE]), r % PAGE], vn[b])
        now = [n + t + 1 for n in kept]
        zero = lambda x: np.nan_to_num(num(x))
        want, want_lse, spread, reach = orc.decode_paged(num(qr), zero(ck), zero(cv), ctable.cpu().numpy(), now)
        check_attention(num(o), num(l), want, want_lse, spread, reach, max(now), dtype, parts=True)
