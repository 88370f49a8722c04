"""Arguments that the steps around a paged cache refuse on the host, before any GPU work (no GPU needed)."""
import pytest
import torch

import paper_2404_14469_amd as pkg

FAKE, ODD = 0x1000, 0x1008      # 16-byte aligned; 8-byte aligned only.  Never dereferenced: validation comes first


def append(**kw):
    a = dict(dtype=0, q=FAKE, k=FAKE, v=FAKE, cu=FAKE, starts=FAKE, pos=FAKE, T=100, B=3, Hq=8, Hkv=2, D=128, qr=1024, qh=128,
             kr=256, kh=128, vr=256, vh=128, cos=FAKE, sin=FAKE, npos=4096, rot=128, inter=0, kp=FAKE, vp=FAKE, table=FAKE, cols=10,
             pages=30, page=16, qo=FAKE, qor=1024, qoh=128, ko=FAKE, kor=256, koh=128)
    assert set(kw) <= set(a)
    a.update(kw)
    return pkg.load().snapkv_append_paged(*a.values(), None)


@pytest.mark.parametrize("kw,code", [
    (dict(T=0), 0), (dict(B=0, cu=None), 0), (dict(T=0, k=None, v=None), 0),
    (dict(dtype=3), -1), (dict(T=-1), -1), (dict(B=-1), -1), (dict(Hkv=0), -1), (dict(Hq=7), -1), (dict(Hq=-1), -1),
    (dict(k=None), -1), (dict(v=None), -1), (dict(starts=None), -1), (dict(kp=None), -1), (dict(vp=None), -1), (dict(table=None), -1),
    (dict(q=None), -1), (dict(qo=None), -1), (dict(Hq=0), -1), (dict(cu=None), -1), (dict(pages=0), -1), (dict(page=0), -1),
    (dict(cols=0), -1), (dict(rot=-16), -1), (dict(rot=144), -1), (dict(inter=2), -1), (dict(cos=None), -1), (dict(sin=None), -1),
    (dict(npos=0), -1), (dict(kr=64), -1), (dict(vh=-128), -1), (dict(qor=8), -1), (dict(koh=-8), -1),
    (dict(D=96, kr=96, rot=96), -2), (dict(D=256), -2), (dict(rot=24), -2), (dict(rot=8), -2), (dict(dtype=1, rot=12), -2),
    (dict(T=1 << 26), -2), (dict(T=1 << 31), -2), (dict(pages=(1 << 31) + 1), -2), (dict(Hq=0, q=None, qo=None, Hkv=40000), -2),
    (dict(q=ODD), -3), (dict(k=ODD), -3), (dict(v=ODD), -3), (dict(qo=ODD), -3), (dict(ko=ODD), -3), (dict(kp=ODD), -3), (dict(vp=ODD), -3),
    (dict(cos=ODD), -3), (dict(sin=ODD), -3), (dict(kr=260), -3), (dict(vh=132), -3), (dict(starts=0x1002), -3), (dict(cu=0x1001), -3),
    (dict(pos=0x1002), -3), (dict(table=0x1002), -3),
])
def test_append_refuses(kw, code):
    assert append(**kw) == code


def prompt(**kw):
    a = dict(dtype=0, q=FAKE, k=FAKE, v=FAKE, cu=FAKE, B=3, T=100, Hq=8, Hkv=2, D=128, qr=1024, qh=128, kr=256, kh=128, vr=256,
             vh=128, out=FAKE, lse=FAKE)
    assert set(kw) <= set(a)
    a.update(kw)
    return pkg.load().snapkv_prompt_attention(*a.values(), None)


@pytest.mark.parametrize("kw,code", [
    (dict(T=0), 0), (dict(B=0), 0), (dict(dtype=-1), -1), (dict(T=-1), -1), (dict(B=-2), -1), (dict(Hq=0), -1), (dict(Hkv=0), -1),
    (dict(Hq=9), -1), (dict(q=None), -1), (dict(k=None), -1), (dict(v=None), -1), (dict(cu=None), -1), (dict(out=None), -1),
    (dict(qr=127), -1), (dict(kh=-1), -1), (dict(dtype=1), -2), (dict(D=96), -2), (dict(D=32), -2), (dict(T=1 << 30), -2),
    (dict(Hq=65536, Hkv=65536), -2), (dict(B=1 << 21), -2), (dict(T=(1 << 30) - 1, Hq=4, Hkv=4), -2), (dict(kr=(1 << 24) + 8), -2), (dict(vr=(1 << 24) + 8), -2), (dict(q=ODD), -3), (dict(k=ODD), -3), (dict(v=ODD), -3), (dict(out=ODD), -3), (dict(lse=0x1002), -3),
    (dict(cu=0x1002), -3), (dict(qr=1028), -3), (dict(vh=4), -3),
])
def test_prompt_attention_refuses(kw, code):
    assert prompt(**kw) == code


def decode(**kw):
    a = dict(dtype=0, q=FAKE, kp=FAKE, vp=FAKE, table=FAKE, cols=400, pages=900, page=16, lens=FAKE, max_len=6000, B=2, Hq=8, Hkv=2,
             D=128, out=FAKE, lse=FAKE, ws=0x10000, ws_bytes=1 << 40)
    assert set(kw) <= set(a)
    a.update(kw)
    return pkg.load().snapkv_decode_attention_paged(*a.values(), None)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=9), -1), (dict(q=None), -1), (dict(kp=None), -1), (dict(vp=None), -1), (dict(table=None), -1), (dict(lens=None), -1),
    (dict(out=None), -1), (dict(B=0), -1), (dict(Hq=0), -1), (dict(Hkv=0), -1), (dict(Hq=9), -1), (dict(pages=0), -1), (dict(page=0), -1),
    (dict(cols=0), -1), (dict(max_len=0), -1), (dict(max_len=6401), -1), (dict(dtype=1), -2), (dict(D=96), -2), (dict(Hq=34), -2),
    (dict(B=65536), -2), (dict(Hq=60000, Hkv=60000, max_len=1 << 20, cols=1 << 20), -2), (dict(B=60000, Hq=512, Hkv=32), -2), (dict(max_len=(1 << 30) + 1, cols=1 << 30), -2), (dict(q=ODD), -3), (dict(kp=ODD), -3), (dict(vp=ODD), -3),
    (dict(out=ODD), -3), (dict(lse=0x1002), -3), (dict(lens=0x1002), -3), (dict(table=0x1002), -3), (dict(ws=0x10010), -3),
    (dict(ws=None), -4), (dict(ws_bytes=100), -4),
])
def test_decode_paged_refuses(kw, code):
    assert decode(**kw) == code


def test_decode_paged_workspace_bytes():
    need = pkg.snapkv_decode_paged_workspace_bytes
    assert need(2, 8, 2, 128, 100) == 0                        # one workgroup per (sequence, KV head)
    assert need(0, 8, 2, 128, 100) == need(2, 9, 2, 128, 9000) == need(2, 8, 2, 96, 9000) == need(2, 8, 2, 128, 0) == 0
    assert 0 < need(1, 8, 2, 128, 9000) < need(1, 8, 2, 128, 90000) and need(1, 8, 2, 64, 9000) < need(1, 8, 2, 128, 9000)


def test_binding_refuses_tensors_of_the_wrong_kind():
    """Shapes, types and places, without a GPU: a tensor on the CPU is refused after the shapes."""
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
    k, pages, table = bf(10, 2, 64), bf(4, 16, 2, 64), i32(3, 2)
    call = pkg.snapkv_append_paged
    for args, kw in [
            ((k, bf(10, 2, 32), pages, pages, table, i32(3)), {}), ((k, k, bf(4, 16, 3, 64), bf(4, 16, 3, 64), table, i32(3)), {}),
            ((k, k, pages, bf(5, 16, 2, 64), table, i32(3)), {}), ((k, k, pages, pages, i32(3), i32(3)), {}),
            ((k, k, pages, pages, table, i32(4)), {}), ((k, k, pages, pages, table, i32(3)), dict(cu_seqlens=i32(3))),
            ((k, k, pages, pages, table, i32(3)), dict(positions=i32(9))), ((k, k, pages, pages, table, i32(3)), dict(cos=torch.zeros(4, 32))),
            ((k, k, pages, pages, table, i32(3)), dict(q=bf(10, 4, 64))), ((k, k, pages, pages, table, i32(3)), dict(q=bf(9, 4, 64), q_out=bf(9, 4, 64))),
            ((k, k, pages, pages, table, i32(3)), dict(k_out=bf(10, 3, 64))), ((k, k, pages, pages, table, i32(3)), dict(cu_seqlens=i32(4)))]:
        with pytest.raises(ValueError):
            call(*args, stream=0, **kw)
    q = bf(10, 4, 64)
    for args in [(q, bf(9, 2, 64), k, i32(2), q), (q, k, bf(10, 1, 64), i32(2), q), (q, k, k, i32(2), bf(10, 4, 32)), (q, k, k, i32(2), q, torch.zeros(10, 4)),
                 (q, k, k, i32(2, 2), q), (q, k, k, i32(2), q)]:
        with pytest.raises(ValueError):
            pkg.snapkv_prompt_attention(*args, stream=0)
    q = bf(3, 4, 64)
    for args in [(bf(3, 4, 32), pages, pages, table, i32(3), 9, q), (q, pages, bf(4, 8, 2, 64), table, i32(3), 9, q), (q, pages, pages, i32(2, 2), i32(3), 9, q),
                 (q, pages, pages, table, i32(2), 9, q), (q, pages, pages, table, i32(3), 9, bf(3, 4, 32)), (q, pages, pages, table, i32(3), 9, q, torch.zeros(4, 3)),
                 (q, pages, pages, table, i32(3), 9, q)]:
        with pytest.raises(ValueError):
            pkg.snapkv_decode_attention_paged(*args, stream=0)
