"""Calls of snapkv_append_paged_mx and snapkv_read_paged_mx so large that their rows go past the caches, against the same work in smaller calls (which other
tests compare with the oracle): the same bits."""
import pytest
import torch

from serve_checks import DT, offsets, seeded, tables
from test_gpu_mx_cache import empty_pool

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("kind", ["fp8", "fp4"])
@pytest.mark.parametrize("dt", ["bf16", "f16", "f32"])
def test_append_of_large_outputs(snapkv, dt, kind, D, inter):
    """Over 500 MB of rotated queries and keys."""
    Hq, Hkv, page, dtype = 40, 20, 16, DT[dt]
    gen, each = seeded(D + inter), 60 * D * torch.finfo(dtype).bits // 8
    T = 510_000_000 // each
    wide = torch.empty((T, (Hq + 2 * Hkv) * D), device="cuda", dtype=dtype).normal_(generator=gen)
    q, k, v = (t.view(T, -1, D) for t in wide.split([Hq * D, Hkv * D, Hkv * D], dim=1))
    pages = -(-T // page)
    table = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32).view(1, -1)
    cos, sin = tables(997, D // 2)
    positions = (torch.arange(T, device="cuda") % 997).to(torch.int32)

    def call(pool, q_out, k_out, a, b):
        snapkv.snapkv_append_paged_mx(k[a:b], v[a:b], *pool, table, torch.tensor([a], dtype=torch.int32, device="cuda"), cu_seqlens=offsets([b - a]),
                                      positions=positions[a:b], cos=cos, sin=sin, interleaved=inter, q=q[a:b], q_out=q_out[a:b], k_out=k_out[a:b])
    made = []
    for step in (T, T // 5):
        made.append((empty_pool(pages, page, Hkv, D, kind), torch.empty((T, Hq, D), device="cuda", dtype=dtype), torch.empty((T, Hkv, D), device="cuda", dtype=dtype)))
        for a in range(0, T, step):
            call(*made[-1], a, min(T, a + step))
    torch.cuda.synchronize()
    (pool, q_out, k_out), (pool2, q_out2, k_out2) = made
    assert all(torch.equal(a, b) for a, b in zip(pool + [q_out, k_out], pool2 + [q_out2, k_out2]))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("kind", ["fp8", "fp4"])
@pytest.mark.parametrize("dt", ["bf16", "f16", "f32"])
def test_read_of_large_outputs(snapkv, dt, kind, D):
    """100 MB of rows."""
    Hkv, page, dtype = 20, 16, DT[dt]
    gen = seeded(D)
    T = 100_000_000 // (2 * Hkv * D * torch.finfo(dtype).bits // 8)
    pages = -(-T // page)
    pool = empty_pool(pages, page, Hkv, D, kind)
    for i, t in enumerate(pool):
        t.copy_(torch.randint(0 if i % 2 == 0 else 110, 256 if i % 2 == 0 else 140, t.shape, generator=gen, device="cuda"))
    table = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32).view(1, -1)
    outs = []
    for step in (T, T // 2 + 1, T // 9):
        outs.append([torch.zeros((Hkv, T, D), device="cuda", dtype=dtype).transpose(0, 1) for _ in range(2)])
        for a in range(0, T, step):
            b = min(T, a + step)
            snapkv.snapkv_read_paged_mx(*pool, table, torch.tensor([a], dtype=torch.int32, device="cuda"), outs[-1][0][a:b], outs[-1][1][a:b], cu_seqlens=offsets([b - a]))
    torch.cuda.synchronize()
    bits = torch.int32 if dt == "f32" else torch.int16                          # (8-bit codes of NaN are among them)
    same = lambda a, b: torch.equal(a.transpose(0, 1).view(bits), b.transpose(0, 1).view(bits))
    assert all(same(a, b) for i in (1, 2) for a, b in zip(outs[0], outs[i]))
