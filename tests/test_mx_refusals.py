"""Arguments that the steps over microscaled pages and over shared prefixes refuse on the host (no GPU needed)."""
import itertools

import pytest
import torch

import paper_2404_14469_amd as pkg

FAKE, ODD = 0x1000, 0x1008      # 16-byte aligned; 8-byte aligned only.  Never dereferenced: validation comes first


def append(**kw):
    a = dict(dtype=0, cache=1, q=FAKE, k=FAKE, v=FAKE, cu=FAKE, starts=FAKE, pos=FAKE, T=100, B=3, Hq=8, Hkv=2, D=128, qr=1024, qh=128,
             kr=256, kh=128, vr=256, vh=128, cos=FAKE, sin=FAKE, npos=4096, rot=128, inter=0, kp=FAKE, ks=FAKE, vp=FAKE, vs=FAKE,
             table=FAKE, cols=10, pages=30, page=16, qo=FAKE, qor=1024, qoh=128, ko=FAKE, kor=256, koh=128)
    assert set(kw) <= set(a)
    a.update(kw)
    return pkg.load().snapkv_append_paged_mx(*a.values(), None)


@pytest.mark.parametrize("kw,code", [
    (dict(T=0), 0), (dict(B=0, cu=None), 0), (dict(cache=0), -1), (dict(cache=3), -1), (dict(cache=-1), -1), (dict(dtype=3), -1),
    (dict(T=-1), -1), (dict(Hkv=0), -1), (dict(Hq=7), -1), (dict(k=None), -1), (dict(kp=None), -1), (dict(ks=None), -1), (dict(vs=None), -1),
    (dict(vp=None), -1), (dict(q=None), -1), (dict(cu=None), -1), (dict(page=0), -1), (dict(cos=None), -1), (dict(rot=144), -1),
    (dict(qor=8), -1), (dict(koh=8), -1), (dict(D=96, kr=96, rot=96), -2), (dict(rot=24), -2), (dict(T=1 << 26), -2), (dict(dtype=1, rot=12), -2),
    (dict(kp=ODD), -3), (dict(ks=ODD), -3), (dict(vs=ODD), -3), (dict(vp=ODD), -3), (dict(q=ODD), -3), (dict(starts=0x1002), -3),
])
def test_append_refuses(kw, code):
    assert append(**kw) == code


def read(**kw):
    a = dict(dtype=0, cache=2, kp=FAKE, ks=FAKE, vp=FAKE, vs=FAKE, table=FAKE, cols=10, pages=30, page=16, cu=FAKE, starts=FAKE, T=100,
             B=3, Hkv=2, D=128, ko=FAKE, kor=256, koh=128, vo=FAKE, vor=256, voh=128)
    assert set(kw) <= set(a)
    a.update(kw)
    return pkg.load().snapkv_read_paged_mx(*a.values(), None)


@pytest.mark.parametrize("kw,code", [
    (dict(T=0), 0), (dict(B=0), 0), (dict(cache=0), -1), (dict(cache=3), -1), (dict(dtype=-1), -1), (dict(T=-1), -1), (dict(B=-1), -1),
    (dict(Hkv=0), -1), (dict(kp=None), -1), (dict(ks=None), -1), (dict(vp=None), -1), (dict(vs=None), -1), (dict(table=None), -1),
    (dict(starts=None), -1), (dict(ko=None), -1), (dict(vo=None), -1), (dict(cu=None), -1), (dict(pages=0), -1), (dict(page=0), -1),
    (dict(cols=0), -1), (dict(kor=64), -1), (dict(voh=-8), -1), (dict(koh=64), -1), (dict(vor=136, voh=128), -1), (dict(D=96), -2),
    (dict(T=1 << 26), -2), (dict(Hkv=40000), -2), (dict(pages=(1 << 31) + 1), -2), (dict(kp=ODD), -3), (dict(ks=ODD), -3),
    (dict(ko=ODD), -3), (dict(vor=260), -3), (dict(starts=0x1002), -3), (dict(cu=0x1002), -3), (dict(table=0x1001), -3),
])
def test_read_refuses(kw, code):
    assert read(**kw) == code


def decode(**kw):
    a = dict(dtype=0, cache=1, q=FAKE, kp=FAKE, ks=FAKE, vp=FAKE, vs=FAKE, table=FAKE, cols=400, pages=900, page=16, lens=FAKE,
             max_len=6000, B=2, Hq=8, Hkv=2, D=128, out=FAKE, lse=FAKE, ws=0x10000, ws_bytes=1 << 40)
    assert set(kw) <= set(a)
    a.update(kw)
    return pkg.load().snapkv_decode_attention_paged_mx(*a.values(), None)


STEP = [
    (dict(dtype=9), -1), (dict(cache=3), -1), (dict(cache=-1), -1), (dict(q=None), -1), (dict(kp=None), -1), (dict(vp=None), -1),
    (dict(table=None), -1), (dict(lens=None), -1), (dict(out=None), -1), (dict(B=0), -1), (dict(Hq=0), -1), (dict(Hkv=0), -1), (dict(Hq=9), -1),
    (dict(pages=0), -1), (dict(page=0), -1), (dict(cols=0), -1), (dict(max_len=0), -1), (dict(max_len=6401), -1), (dict(ks=None), -1),
    (dict(vs=None), -1), (dict(dtype=1), -2), (dict(D=96), -2), (dict(Hq=34), -2), (dict(B=65536), -2),
    (dict(max_len=(1 << 30) + 1, cols=1 << 30), -2), (dict(q=ODD), -3), (dict(kp=ODD), -3), (dict(ks=ODD), -3), (dict(vp=ODD), -3),
    (dict(vs=ODD), -3), (dict(out=ODD), -3), (dict(lse=0x1002), -3), (dict(lens=0x1002), -3), (dict(table=0x1002), -3), (dict(ws=0x10010), -3),
    (dict(ws=None), -4), (dict(ws_bytes=100), -4)]


@pytest.mark.parametrize("kw,code", STEP + [(dict(cache=0), -1), (dict(cache=0, ks=None, vs=None), -1)])
def test_decode_refuses(kw, code):
    assert decode(**kw) == code


def shared(**kw):
    a = dict(dtype=0, cache=1, q=FAKE, kp=FAKE, ks=FAKE, vp=FAKE, vs=FAKE, pages=900, page=16, cu=FAKE, G=2, pt=FAKE, pcols=400, pl=FAKE,
             max_prefix=6000, table=FAKE, cols=400, lens=FAKE, max_len=6000, B=4, Hq=8, Hkv=2, D=128, out=FAKE, lse=FAKE, ws=0x10000,
             ws_bytes=1 << 40)
    assert set(kw) <= set(a)
    a.update(kw)
    return pkg.load().snapkv_decode_attention_shared(*a.values(), None)


@pytest.mark.parametrize("kw,code", STEP + [
    (dict(cache=0), -1), (dict(cache=0, ks=None), -1), (dict(cache=0, vs=None), -1), (dict(pt=None), -1), (dict(pl=None), -1), (dict(pcols=0), -1),
    (dict(G=0), -1), (dict(G=5), -1), (dict(cu=None), -1), (dict(max_prefix=0), -1), (dict(max_prefix=6401), -1),
    (dict(max_prefix=(1 << 30) + 1, pcols=1 << 30), -2), (dict(B=65535, Hkv=17, Hq=17), -2), (dict(G=4, Hkv=32, Hq=32, max_prefix=1 << 30, pcols=1 << 30), -2),
    (dict(cu=0x1002), -3), (dict(pt=0x1002), -3), (dict(pl=0x1001), -3)])
def test_shared_refuses(kw, code):
    assert shared(**kw) == code


def test_one_group_needs_no_offsets():
    assert shared(G=1, cu=None, ws=None) == -4 and shared(cache=0, ks=None, vs=None, ws=None) == -4


def test_workspaces():
    need = pkg.snapkv_decode_paged_mx_workspace_bytes
    assert need(2, 8, 2, 128, 100) == 0
    assert need(0, 8, 2, 128, 100) == need(2, 9, 2, 128, 9000) == need(2, 8, 2, 96, 9000) == need(2, 8, 2, 128, 0) == 0
    assert 0 < need(1, 8, 2, 128, 9000) < need(1, 8, 2, 128, 90000)
    need = pkg.snapkv_decode_shared_workspace_bytes
    assert need(2, 3, 8, 2, 128, 100, 100) == need(2, 0, 8, 2, 128, 100, 100) == need(2, 1, 8, 2, 128, 0, 100) == need(2, 1, 8, 2, 80, 9, 9) == 0
    for B, (Hq, Hkv), D, longest in itertools.product([1, 2, 7, 32, 100, 1000, 30000], [(1, 1), (32, 8), (32, 32), (16, 1)], [64, 128], [1, 513, 131072, 1 << 20]):
        for G in {1, max(1, B // 3), B}:
            n = need(B, G, Hq, Hkv, D, longest, 300)
            if G * Hkv * longest > 1 << 36:
                assert n == 0
                continue
            # at most 256 shares of a prefix, as many as give 1024 workgroups, and 7 (or few sequences' more) of own rows
            units = (G + B * (Hq // Hkv) // 64) * Hkv
            shares = min(256, (longest + 127) // 128, 1024 // units + 1) + 7 + 16384 // (B * Hkv)
            assert 0 < n <= B * Hq * shares * (4 * D + 8) + 256, (B, G, Hq, Hkv, D, longest)


def test_binding_refuses_tensors_of_the_wrong_kind():
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)
    u8 = lambda *s: torch.zeros(s, dtype=torch.uint8)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
    k, codes, scales, table = bf(10, 2, 64), u8(4, 16, 2, 64), u8(4, 16, 2, 2), i32(3, 2)
    half = u8(4, 16, 2, 32)
    pools = [(codes, scales, half, scales), (codes, u8(4, 16, 2, 4), codes, scales), (codes, scales, codes, u8(4, 16, 2)),
             (u8(4, 16, 2, 48), scales, u8(4, 16, 2, 48), scales), (u8(4, 16, 1, 64), scales, u8(4, 16, 1, 64), scales)]
    good = (codes, scales, codes, scales)
    for pool in pools + [good]:             # (the last: on the CPU)
        with pytest.raises(ValueError):
            pkg.snapkv_append_paged_mx(k, k, *pool, table, i32(3), stream=0)
        with pytest.raises(ValueError):
            pkg.snapkv_read_paged_mx(*pool, table, i32(3), k, k, stream=0)
        with pytest.raises(ValueError):
            pkg.snapkv_decode_attention_paged_mx(bf(3, 4, 64), *pool, table, i32(3), 9, bf(3, 4, 64), stream=0)
        with pytest.raises(ValueError):
            pkg.snapkv_decode_attention_shared(bf(3, 4, 64), pool[0], pool[2], i32(1, 2), i32(1), 9, table, i32(3), 9, bf(3, 4, 64),
                                               k_scales=pool[1], v_scales=pool[3], stream=0)
    for kw in (dict(cu_seqlens=i32(3)), dict(positions=i32(9)), dict(cos=torch.zeros(4, 32)), dict(q=bf(10, 4, 64)), dict(k_out=bf(10, 3, 64))):
        with pytest.raises(ValueError):
            pkg.snapkv_append_paged_mx(k, k, *good, table, i32(3), stream=0, **kw)
    for args in ((table, i32(4), k, k), (i32(3), i32(3), k, k), (table, i32(3), k, bf(9, 2, 64)), (table, i32(3), k, k.float())):
        with pytest.raises(ValueError):
            pkg.snapkv_read_paged_mx(*good, *args, stream=0)
    q, pages = bf(3, 4, 64), bf(4, 16, 2, 64)
    ok = dict(q=q, k_pages=pages, v_pages=pages, prefix_table=i32(1, 2), prefix_lens=i32(1), max_prefix=9, block_table=table, lens=i32(3), max_len=9, out=q)
    for kw in (dict(), dict(q=bf(3, 4, 32)), dict(v_pages=bf(4, 8, 2, 64)), dict(prefix_table=i32(2)), dict(prefix_table=i32(2, 2)), dict(prefix_lens=i32(2)),
               dict(cu_groups=i32(3)), dict(prefix_table=i32(2, 2), prefix_lens=i32(2)), dict(block_table=i32(2, 2)), dict(lens=i32(2)),
               dict(out=bf(3, 4, 32)), dict(out_lse=torch.zeros(4, 3)), dict(k_scales=scales), dict(k_pages=codes, v_pages=codes)):
        with pytest.raises(ValueError):
            pkg.snapkv_decode_attention_shared(**{**ok, **kw}, stream=0)
