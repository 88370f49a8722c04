"""Steps whose sequences can be long or many: workgroups that take four, two or one KV heads, and rows fetched past the caches."""
import pytest
import torch

from mx_checks import mx_pool
from serve_checks import DT, rows, seeded
from test_gpu_mx_decode import check, run
from test_gpu_shared_prefix import build
from test_gpu_shared_prefix import check as check_shared
from test_gpu_shared_prefix import run as run_shared

pytestmark = pytest.mark.gpu

CASES = [   # lens, page, Hq, Hkv, D, dtype: sequences x KV heads x longest is 2^20 at least
    ([1900] + [3] * 190, 16, 3, 3, 128, "bf16"),            # one head
    ([3000, 0, 2700] + [1, 33, 130] * 60, 24, 4, 2, 128, "f16"),       # two
    ([3000, 0, 2700] + [1, 33, 130] * 60, 24, 12, 6, 64, "bf16"),      # two of six
    ([2100, 2047, 513] + [129, 31, 0, 512] * 40, 1, 16, 4, 128, "bf16"),
    ([2100, 2047, 513] + [129, 31, 0, 512] * 40, 7, 32, 8, 64, "f16"),
    ([1500] + [16, 17, 63, 64, 65] * 18, 128, 12, 12, 128, "f16"),
]


@pytest.mark.parametrize("kind", ["fp8", "fp4"])
@pytest.mark.parametrize("n", range(len(CASES)))
def test_step_matches_oracle(snapkv, n, kind):
    lens, page, Hq, Hkv, D, dt = CASES[n]
    assert len(lens) * Hkv * max(lens) >= 1 << 20
    gen = seeded(1300 + n)
    q = rows(gen, len(lens), Hq, D, DT[dt], "tokens")
    pool, table = mx_pool(gen, lens, page, Hkv, D, kind)
    dl = torch.tensor(lens, dtype=torch.int32, device="cuda")
    out, lse = run(snapkv, q, pool, table, dl, max(lens))
    check(q, pool, kind, table, lens, out, lse)
    again, _ = run(snapkv, q, pool, table, dl, max(lens), lse=False)
    assert torch.equal(out, again)


@pytest.mark.parametrize("kind", ["fp8", "fp4", "plain"])
@pytest.mark.parametrize("groups", [[40, 2, 60], [102]])
def test_shared_step_matches_oracle(snapkv, groups, kind):
    lens = [(7 * i) % 90 for i in range(101)] + [2600]
    assert len(lens) * 4 * max(lens) >= 1 << 20
    s = build(seeded(1350), [300 + 77 * i for i in range(len(groups))], groups, lens, 16, 8, 4, 128, torch.bfloat16, kind)
    check_shared(s, kind, *run_shared(snapkv, s))


@pytest.mark.parametrize("room, kind", [(0, "plain"), (300, "plain"), (1200, "plain"), (300, "fp8"), (1200, "fp4")])
@pytest.mark.parametrize("Hq", [128, 64])
def test_shares_of_wide_tiles(snapkv, Hq, room, kind):
    """Tiles of 128 and 64 query heads, their prefixes cut into 32, 24 or 16 shares as own rows may be few, as many or more; the last
    shares of both prefixes are empty or partial."""
    lens = [(3 * i) % 11 for i in range(16)]
    s = build(seeded(1370), [4200, 3001], [8, 8], lens, 16, Hq, 8, 128, torch.bfloat16, kind, room=room)
    keys, met = 16 * 8 * s["max_len"], 2 * 8 * 4200                # of own rows; of prefixes, one tile to a group and KV head
    assert (keys < 0.3 * met, keys >= 1.5 * met) == (room == 0, room == 1200)
    check_shared(s, kind, *run_shared(snapkv, s))
    out, lse = run_shared(snapkv, s)
    again, _ = run_shared(snapkv, s, lse=False)
    assert torch.equal(out, again)


@pytest.mark.parametrize("members", [3, 20])
def test_prefixes_of_many_kv_heads(snapkv, members):
    """So many tiles and KV heads (160) that prefixes are cut into a few shares only, with tiles of 16 and of 64 query heads."""
    groups = [members, members + 1, 1, members, members - 1]
    s = build(seeded(1380), [700, 129, 1001, 64, 513], groups, [i % 9 for i in range(sum(groups))], 16, 96, 32, 64, torch.bfloat16, "plain")
    check_shared(s, "plain", *run_shared(snapkv, s))


def test_a_block_of_nan_reaches_its_own_heads_only(snapkv):
    """Scales of four KV heads are fetched together: a NaN of one head's leaves the others' bits as they are."""
    gen, lens = seeded(1360), [2100] + [500] * 130
    q = rows(gen, len(lens), 8, 128, torch.bfloat16, "tokens")
    pool, table = mx_pool(gen, lens, 16, 4, 128, "fp8")
    dl = torch.tensor(lens, dtype=torch.int32, device="cuda")
    want = run(snapkv, q, pool, table, dl, 2100)
    pool[1][table[0, 70].long(), 5, 2, 3] = 255                     # a key of KV head 2
    pool[3][table[5, 20].long(), 9, 1, 0] = 255                     # a value of KV head 1, elements 0 .. 31
    got = run(snapkv, q, pool, table, dl, 2100)
    torch.cuda.synchronize()
    same = torch.ones((len(lens), 8), dtype=torch.bool, device="cuda")
    same[0, 4:6] = False
    assert got[0][~same].isnan().all() and got[1][~same].isnan().all()
    assert torch.equal(got[1][same], want[1][same])
    same[5, 2:4] = False
    assert torch.equal(got[0][same], want[0][same])
    assert got[0][5, 2:4, :32].isnan().all() and torch.equal(got[0][5, 2:4, 32:], want[0][5, 2:4, 32:])
