"""snapkv_decode_attention_shared against the fp64 oracle; bounds in mx_checks.py."""
import numpy as np
import pytest
import torch

from mx_checks import check_step, mx_pool, mx_values
from oracle import mx_oracle as orc
from serve_checks import DT, fill_rows, num, offsets, pool, rows, seeded

pytestmark = pytest.mark.gpu


def build(gen, prefixes, groups, lens, page, Hq, Hkv, D, dtype, kind, before=0, room=0):
    """Inputs of a step: `groups` sequences of each prefix, `before` sequences ahead of the first group; lens of all sequences."""
    spans = list(prefixes) + [n + room for n in lens]
    s = dict(q=rows(gen, len(lens), Hq, D, dtype, "tokens"))
    if kind == "plain":
        s["k_pages"], s["v_pages"], table = pool(gen, spans, page, Hkv, D, dtype)
        fill_rows(gen, s["k_pages"], s["v_pages"], table, list(prefixes) + list(lens))
    else:
        (s["k_pages"], s["k_scales"], s["v_pages"], s["v_scales"]), table = mx_pool(gen, spans, page, Hkv, D, kind)
        for b, n in enumerate(lens):
            j = torch.arange(n, n + room, device="cuda")
            for t in (s["k_scales"], s["v_scales"]):
                t[table[len(prefixes) + b, j // page].long(), j % page] = 255
    G = len(prefixes)
    s.update(prefix_table=table[:G].contiguous(), block_table=table[G:].contiguous(), max_prefix=max(max(prefixes), 1), max_len=max(max(lens), 1) + room,
             prefix_lens=torch.tensor(prefixes, dtype=torch.int32, device="cuda"), lens=torch.tensor(lens, dtype=torch.int32, device="cuda"),
             cu_groups=offsets(groups, before))
    return s


def run(snapkv, s, lse=True, **kw):
    out = torch.full(s["q"].shape, 77.0, device="cuda", dtype=s["q"].dtype)
    out_lse = torch.full(s["q"].shape[:2], 77.0, device="cuda") if lse else None
    snapkv.snapkv_decode_attention_shared(**s, out=out, out_lse=out_lse, **kw)
    return out, out_lse


def check(s, kind, out, lse):
    torch.cuda.synchronize()
    cpu = lambda n: s[n].cpu().numpy()
    if kind == "plain":
        k, v = (np.nan_to_num(num(s[n])) for n in ("k_pages", "v_pages"))
    else:
        k, v = (mx_values(s[n + "_pages"], s[n + "_scales"], kind) for n in ("k", "v"))
    cu = cpu("cu_groups")
    pl, ln = np.clip(cpu("prefix_lens"), 0, s["max_prefix"]), np.clip(cpu("lens"), 0, s["max_len"])
    want = orc.decode_shared(num(s["q"]), k, v, cpu("prefix_table"), pl, cpu("block_table"), ln, list(zip(cu[:-1], cu[1:])))
    check_step(out, lse, *want, int(pl.max() + ln.max()) + 1, s["q"].dtype, plain=kind == "plain",
               rounded=s["q"].shape[0] * s["q"].shape[1] // s["k_pages"].shape[2] > 32 * len(pl))


CASES = [   # prefixes, groups, lens, page, Hq, Hkv, D, dtype, kind, before
    ([1], [1], [1], 16, 4, 4, 128, "bf16", "plain", 0),
    ([2048], [2], [3, 3], 16, 32, 8, 128, "bf16", "plain", 0),
    ([130, 0, 33, 700], [3, 2, 0, 4], [0, 1, 17, 5, 0, 33, 2, 1, 64], 16, 8, 2, 64, "bf16", "plain", 0),
    ([500, 129], [5, 9], [1, 333, 700, 64, 129, 17, 1025, 2, 450, 90, 300, 15, 33, 511, 60, 0, 1], 16, 4, 4, 64, "f16", "plain", 1),
    ([1000], [33], [i % 7 for i in range(33)], 24, 8, 2, 128, "bf16", "plain", 0),      # 132 rows: tiles of 64 and what is left
    ([1000], [16], [1] * 16, 8, 16, 1, 128, "f16", "plain", 0),                         # 256 rows of one KV head
    ([257, 4000], [17, 3], [40 + i for i in range(20)], 1, 6, 2, 128, "bf16", "plain", 0),
    ([2113], [2], [5, 0], 16, 32, 8, 128, "bf16", "fp8", 0),
    ([513, 100], [7, 12], [3 * i for i in range(19)], 7, 8, 4, 64, "f16", "fp8", 0),
    ([900], [40], [1 + 3 * i for i in range(40)], 32, 8, 2, 128, "f16", "fp4", 0),
    ([900, 31, 1], [1, 1, 1], [100, 0, 7], 16, 3, 3, 128, "bf16", "fp4", 0),
    ([1500], [70], [i % 3 for i in range(70)], 128, 2, 2, 64, "bf16", "fp4", 0),
    ([64] * 70, [2] * 70, [2] * 141, 16, 2, 1, 64, "bf16", "plain", 1),                 # more groups than lanes
    ([600, 600, 600], [1, 30, 2], [9] * 33, 16, 12, 4, 128, "bf16", "plain", 0),        # groups of very different size
]


@pytest.mark.parametrize("n", range(len(CASES)))
def test_step_matches_oracle(snapkv, n):
    prefixes, groups, lens, page, Hq, Hkv, D, dt, kind, before = CASES[n]
    s = build(seeded(1500 + n), prefixes, groups, lens, page, Hq, Hkv, D, DT[dt], kind, before)
    out, lse = run(snapkv, s)
    check(s, kind, out, lse)
    again, _ = run(snapkv, s, lse=False)
    assert torch.equal(out, again)


@pytest.mark.parametrize("kind", ["plain", "fp8", "fp4"])
@pytest.mark.parametrize("members", [1, 3, 4, 5, 8, 9, 16, 17, 31, 32, 33, 65])
def test_tiles_of_query_heads(snapkv, members, kind):
    """Group sizes around whole tiles, four query heads to a KV head; a prefix that ends inside a step, a page and a share."""
    s = build(seeded(70 + members), [389], [members], [members % 5] * members, 16, 4, 1, 128, torch.bfloat16, kind, room=600)
    check(s, kind, *run(snapkv, s))


@pytest.mark.parametrize("kind", ["plain", "fp8", "fp4"])
@pytest.mark.parametrize("members", [3, 9, 20, 40])
def test_tiles_of_query_heads_of_64_elements(snapkv, members, kind):
    s = build(seeded(170 + members), [643], [members], [1 + members % 4] * members, 24, 8, 2, 64, torch.float16, kind)
    check(s, kind, *run(snapkv, s))


@pytest.mark.parametrize("P", [1, 31, 32, 33, 63, 64, 65, 127, 128, 129, 191, 1000])
@pytest.mark.parametrize("members", [10, 20])
def test_short_prefixes_of_many(snapkv, members, P):
    """Prefixes that end inside a tile and a block of 32 keys, met by tiles of 64 and of 128 query heads."""
    s = build(seeded(200 + P), [P], [members], [1] * members, 16, 8, 2, 128, torch.bfloat16, "plain")
    check(s, "plain", *run(snapkv, s))


def test_one_group_without_offsets(snapkv):
    s = build(seeded(80), [700], [6], [1, 2, 3, 0, 50, 6], 16, 8, 2, 128, torch.bfloat16, "plain")
    out, lse = run(snapkv, s)
    check(s, "plain", out, lse)
    cu = s.pop("cu_groups")
    again, lse2 = run(snapkv, s)
    assert torch.equal(out, again) and torch.equal(lse, lse2)
    s["cu_groups"] = cu


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_prefix_or_own_rows_far_from_the_others(snapkv, dtype):
    """Logits of the prefix far above those of the own rows, and far below."""
    for sign in (1, -1):
        s = build(seeded(81), [600], [5], [40, 1, 300, 7, 90], 16, 4, 2, 128, DT[dtype], "plain")
        s["q"].copy_(s["q"].abs() + 0.5)
        j = torch.arange(600, device="cuda")
        s["k_pages"][s["prefix_table"][0, j // 16].long(), j % 16] += 3 * sign
        check(s, "plain", *run(snapkv, s))


def test_lengths_offsets_and_entries_are_clamped(snapkv):
    s = build(seeded(82), [200, 100], [2, 2], [50] * 4, 16, 4, 2, 64, torch.bfloat16, "plain")
    for t in ("k_pages", "v_pages"):
        s[t].nan_to_num_(0.5)
    s["prefix_lens"].copy_(torch.tensor([1 << 30, -7]))
    s["lens"].copy_(torch.tensor([-1, 1 << 30, 20, 0]))
    s["prefix_table"][0, 2], s["block_table"][1, 0] = 1 << 30, -5
    check(s, "plain", *run(snapkv, s))


def test_nan_stays_with_those_who_see_it(snapkv):
    s = build(seeded(83), [300, 300], [3, 3], [20] * 6, 16, 4, 2, 128, torch.bfloat16, "plain")
    want = run(snapkv, s)
    s["q"][1, 2, 5] = float("nan")                                          # one head of one sequence
    s["v_pages"][s["block_table"][4, 0].long(), 3, 0] = float("nan")        # an own row of sequence 4, KV head 0
    got = run(snapkv, s)
    torch.cuda.synchronize()
    bad = torch.zeros((6, 4), dtype=torch.bool, device="cuda")
    bad[1, 2], bad[4, :2] = True, True
    assert got[0][bad].isnan().all() and torch.equal(got[0][~bad], want[0][~bad])
    assert bool(got[1][1, 2].isnan()) and torch.equal(got[1][~bad], want[1][~bad]) and torch.equal(got[1][4], want[1][4])
    s["k_pages"][s["prefix_table"][0, 2].long(), 3, 1] = float("nan")       # a row of the first prefix, KV head 1
    got = run(snapkv, s)
    torch.cuda.synchronize()
    bad[:3, 2:] = True
    assert got[0][bad].isnan().all() and torch.equal(got[0][~bad], want[0][~bad])


@pytest.mark.parametrize("members", [12, 30])
def test_nan_stays_with_those_who_see_it_in_wide_tiles(snapkv, members):
    s = build(seeded(183), [300, 300], [members, members], [20] * (2 * members), 16, 4, 2, 128, torch.bfloat16, "plain")
    s["q"].mul_(2)
    want = run(snapkv, s)
    s["q"][1, 2, 5] = float("nan")
    got = run(snapkv, s)
    torch.cuda.synchronize()
    bad = torch.zeros((2 * members, 4), dtype=torch.bool, device="cuda")
    bad[1, 2] = True
    assert got[0][bad].isnan().all() and torch.equal(got[0][~bad], want[0][~bad]) and torch.equal(got[1][~bad], want[1][~bad])
    s["v_pages"][s["prefix_table"][0, 2].long(), 3, 1, 70] = float("inf")   # one element of a value of the first prefix, KV head 1
    got = run(snapkv, s)
    torch.cuda.synchronize()
    assert torch.equal(got[1][~bad], want[1][~bad])
    bad[:members, 2:] = True
    assert torch.equal(got[0][~bad], want[0][~bad])
    seen = got[0][:members, 2:].clone()
    assert (seen[..., 70].isinf() | seen[..., 70].isnan()).all()
    seen[..., 70] = want[0][:members, 2:, 70]
    keep = torch.ones((members, 2), dtype=torch.bool, device="cuda")
    keep[1, 0] = False
    assert torch.equal(seen[keep], want[0][:members, 2:][keep])
    s["k_pages"][s["prefix_table"][1, 18].long(), 11, 0] = float("nan")     # the last row of the second prefix, KV head 0
    got = run(snapkv, s)
    torch.cuda.synchronize()
    assert got[0][members:, :2].isnan().all() and torch.equal(got[0][:members, :2], want[0][:members, :2]) and torch.equal(got[0][members:, 2:], want[0][members:, 2:])


def test_fp16_values_near_the_largest(snapkv):
    """A mean of finite numbers is finite."""
    s = build(seeded(184), [400], [12], [0] * 12, 16, 8, 2, 64, torch.float16, "plain")
    s["v_pages"].fill_(65504.0)
    out, _ = run(snapkv, s)
    torch.cuda.synchronize()
    assert out.isfinite().all() and (out.float() >= 65504 * (1 - 2.0 ** -9)).all()


def test_a_prefix_shared_is_the_prefix_of_each(snapkv):
    """Against the step over pages whose tables name the prefix's pages for every sequence."""
    page, P = 16, 1600
    s = build(seeded(84), [P], [9], [1 + 37 * i for i in range(9)], page, 8, 2, 128, torch.bfloat16, "plain")
    out, lse = run(snapkv, s)
    table = torch.cat([s["prefix_table"][:, :P // page].expand(9, -1), s["block_table"]], dim=1).contiguous()
    want, want_lse = torch.empty_like(out), torch.empty_like(lse)
    snapkv.snapkv_decode_attention_paged(s["q"], s["k_pages"], s["v_pages"], table, s["lens"] + P, s["max_len"] + P, want, want_lse)
    torch.cuda.synchronize()
    assert (lse - want_lse).abs().max() <= 1e-4
    assert ((out.double() - want.double()).abs() <= 2.0 ** -7 * want.abs() + 2.0 ** -11).all()


@pytest.mark.parametrize("kind", ["plain", "fp8"])
@pytest.mark.parametrize("members", [3, 24, 60])
def test_pool_beyond_32_bit_offsets(snapkv, members, kind):
    """The same rows behind tables whose pages lie at both ends of a pool of over 4 GiB: the same bits, with tiles of 16, 64 and 128."""
    page, Hkv, D = 128, 16, 128
    s = build(seeded(87), [900], [members], [5, 130, 1] * (members // 3), page, 2 * Hkv, Hkv, D, torch.bfloat16, kind)
    want = run(snapkv, s)
    used = s["k_pages"].shape[0]
    row = s["k_pages"][0].numel() * s["k_pages"].element_size()
    pages = (1 << 32) // row + 2 * used
    moved = torch.arange(used, device="cuda")
    moved = torch.where(moved % 2 == 0, moved, pages - 1 - moved)
    big = dict(s)
    for n in ("k_pages", "v_pages", "k_scales", "v_scales"):
        if n in s:
            big[n] = torch.empty((pages,) + s[n].shape[1:], device="cuda", dtype=s[n].dtype)
            big[n][moved] = s[n]
    for n in ("prefix_table", "block_table"):
        big[n] = torch.where(s[n] < used, moved[s[n].clamp(max=used - 1).long()], s[n]).to(torch.int32)
    assert int(big["prefix_table"][0, :8].max()) * row > 1 << 32 and int(big["prefix_table"][0, :8].min()) < used
    got = run(snapkv, big)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_workspaces_hold_nothing_between_calls(snapkv):
    """A workspace full of NaN, and captured steps of two shapes that share one, replayed with other lengths and groups."""
    gen = seeded(85)
    sets = [build(gen, [900, 300], [3, 4], [20, 5, 0, 700, 1, 2, 3], 16, 8, 2, 128, torch.bfloat16, "plain"),
            build(gen, [3000], [20], [5] * 20, 16, 8, 2, 128, torch.float16, "fp8")]
    size = lambda s: snapkv.snapkv_decode_shared_workspace_bytes(s["q"].shape[0], s["prefix_lens"].shape[0], s["q"].shape[1], s["k_pages"].shape[2], 128, s["max_prefix"], s["max_len"])
    ws = torch.full((max(size(s) for s in sets),), 255, dtype=torch.uint8, device="cuda")
    for s in sets:
        want = run(snapkv, s)
        ws.fill_(255)
        got = run(snapkv, s, workspace=ws)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    graphs, outs = [], []
    torch.cuda.synchronize()
    for s in sets:
        o = (torch.empty_like(s["q"]), torch.empty(s["q"].shape[:2], device="cuda"))
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            snapkv.snapkv_decode_attention_shared(**s, out=o[0], out_lse=o[1], workspace=ws)
        outs.append(o)
    for rep in range(4):
        for s in sets:
            s["q"].normal_(generator=gen)
            s["lens"].copy_((s["lens"] - 1).clamp_(min=0))
            s["prefix_lens"].sub_(111 * rep)
        sets[0]["cu_groups"].copy_(torch.tensor([rep, 2 + rep, 7 - rep % 2]))
        want = [run(snapkv, s) for s in sets]
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            assert torch.equal(o[0], w[0]) and torch.equal(o[1], w[1])
        check(sets[0], "plain", *outs[0])


def test_steps_on_two_streams_with_their_own_workspaces(snapkv):
    gen, sets, want = seeded(86), [], []
    for kind in ("plain", "fp4"):
        s = build(gen, [2000], [12], [33] * 12, 16, 8, 2, 128, torch.bfloat16, kind)
        sets.append((s, torch.empty(snapkv.snapkv_decode_shared_workspace_bytes(12, 1, 8, 2, 128, 2000, 33), dtype=torch.uint8, device="cuda")))
        want.append(run(snapkv, s))
    streams = [torch.cuda.Stream() for _ in sets]
    outs = [[(torch.empty_like(s["q"]), torch.empty((12, 8), device="cuda")) for _ in range(10)] for s, _ in sets]
    torch.cuda.synchronize()
    for i in range(10):
        for (s, ws), st, o in zip(sets, streams, outs):
            snapkv.snapkv_decode_attention_shared(**s, out=o[i][0], out_lse=o[i][1], workspace=ws, stream=st)
    torch.cuda.synchronize()
    for w, o in zip(want, outs):
        assert all(torch.equal(a, w[0]) and torch.equal(b, w[1]) for a, b in o)
    with pytest.raises(ValueError, match="workspace"):
        snapkv.snapkv_decode_attention_shared(**sets[0][0], out=outs[0][0][0], stream=streams[0])
