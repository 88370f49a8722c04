"""snapkv_append_paged finds a token's sequence among many: short, empty, with tokens in front of the first and behind the last."""
import numpy as np
import pytest
import torch

from serve_checks import offsets, rows, seeded

pytestmark = pytest.mark.gpu


def call(snapkv, lengths, first, last, page=4, Hkv=1, D=64, seed=0):
    """Rows into pages and where each token should have gone: slots of -1 for tokens of no sequence."""
    gen, B = seeded(seed), len(lengths)
    T = first + sum(lengths) + last
    k = rows(gen, T, Hkv, D, torch.bfloat16, "tokens")
    starts = torch.randint(0, 6, (B,), generator=gen, device="cuda")
    n = torch.tensor(lengths, device="cuda")
    columns = (6 + max(lengths)) // page + 1
    table = torch.randperm(B * columns, generator=gen, device="cuda").view(B, columns)
    kp = torch.zeros((B * columns, page, Hkv, D), device="cuda", dtype=torch.bfloat16)
    vp, k_out = torch.zeros_like(kp), torch.full_like(k, 9.0)
    cu = offsets(lengths, first)
    snapkv.snapkv_append_paged(k, k, kp, vp, table.to(torch.int32), starts.to(torch.int32), cu_seqlens=cu, k_out=k_out)
    torch.cuda.synchronize()
    seq = torch.arange(B, device="cuda").repeat_interleave(n)
    row = starts[seq] + first + torch.arange(sum(lengths), device="cuda") - cu[seq].long()
    slot = table[seq, row // page] * page + row % page
    mine = slice(first, first + sum(lengths))
    want = torch.zeros_like(kp)
    want.view(-1, Hkv, D)[slot] = k[mine]
    assert torch.equal(kp, want) and torch.equal(vp, want)
    assert torch.equal(k_out[mine], k[mine])
    assert (k_out[:first] == 9).all() and (k_out[first + sum(lengths):] == 9).all()


LENGTHS = {
    "64": [1, 0, 3, 2] * 16, "65": [2] * 65, "one of many": [0] * 700 + [5] + [0] * 3000, "first": [7] + [0] * 4095, "last": [0] * 4096 + [7],
    "empty at the search's borders": [0 if i % 64 in (0, 1, 63) else 1 + i % 3 for i in range(4096)],
    "empty pieces": ([0] * 64 + [1] * 64) * 40, "4097": [1] * 4097, "66 x 66": [i % 4 for i in range(4356)],
}


@pytest.mark.parametrize("first,last", [(0, 0), (37, 5)])
@pytest.mark.parametrize("name", LENGTHS)
def test_every_token_goes_to_its_sequence(snapkv, name, first, last):
    call(snapkv, LENGTHS[name], first, last, seed=len(name))


def test_few_tokens_of_many_sequences(snapkv):
    """Below 1024 tokens the heads of a token are shared out over waves."""
    lengths = [0] * 5000
    for i in np.random.default_rng(3).choice(5000, 300, replace=False):
        lengths[i] = 1 + int(i) % 3
    call(snapkv, lengths, 3, 4, Hkv=12, D=128, seed=1)


def test_the_search_is_short(snapkv):
    """2^18 sequences of a token each: the offsets cost little beside the same call without them."""
    B, page = 1 << 18, 16
    k = rows(seeded(2), B, 1, 64, torch.bfloat16, "tokens")
    kp = torch.zeros((B // page, page, 1, 64), device="cuda", dtype=torch.bfloat16)
    vp = torch.zeros_like(kp)
    at = torch.arange(B, device="cuda", dtype=torch.int32)
    table, starts, cu = (at // page)[:, None].contiguous(), at % page, torch.arange(B + 1, device="cuda", dtype=torch.int32)

    def time(**kw):
        times = []
        for _ in range(4):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            snapkv.snapkv_append_paged(k, k, kp, vp, table, starts, **kw)
            b.record()
            torch.cuda.synchronize()
            times.append(a.elapsed_time(b))
        return min(times)

    plain, searched = time(), time(cu_seqlens=cu)
    assert torch.equal(kp.view(B, 1, 64), k)
    print(f"{plain * 1e3:.0f} us without offsets, {searched * 1e3:.0f} us with")
    assert searched < 20 * plain + 0.2
