"""Which shapes the step over pages takes, and how much workspace it asks for (no GPU needed: the step is called with a length array
at an odd address, which it refuses after the shape)."""
import itertools

import pytest

import paper_2404_14469_amd as pkg

FAKE = 0x1000


def step(B, Hq, Hkv, D, max_len):
    return pkg.load().snapkv_decode_attention_paged(0, FAKE, FAKE, FAKE, FAKE, 1 << 30, 900, 16, FAKE + 2, max_len, B, Hq, Hkv, D, FAKE,
                                                    None, 0x10000, 1 << 60, None)


@pytest.mark.parametrize("B,Hq,Hkv,D,max_len", [
    (1, 34, 2, 128, 9000), (65536, 8, 8, 128, 9000), (2, 65536, 65536, 64, 9000), (60000, 512, 32, 128, 9000), (60000, 320, 20, 128, 9000),
    (64, 65535, 65535, 64, 100), (1, 8, 8, 96, 9000), (1, 8, 8, 128, (1 << 30) + 1), (2, 60000, 60000, 128, 1 << 20), (64, 8, 8, 128, 1 << 30)])
def test_shapes_that_the_step_refuses_need_no_workspace(B, Hq, Hkv, D, max_len):
    assert step(B, Hq, Hkv, D, max_len) == -2
    assert pkg.snapkv_decode_paged_workspace_bytes(B, Hq, Hkv, D, max_len) == 0


def test_shapes_that_it_takes_need_a_bounded_workspace():
    """At most seven partials of a query head, or 16384 of a KV head's query heads in all."""
    for B, (Hq, Hkv), D, max_len in itertools.product([1, 2, 7, 32, 100, 128, 256, 1000, 4096, 30000], [(1, 1), (32, 8), (32, 32), (16, 1), (20, 20)],
                                                      [64, 128], [1, 511, 513, 4096, 9001, 131072, 1 << 20, 1 << 22]):
        need = pkg.snapkv_decode_paged_workspace_bytes(B, Hq, Hkv, D, max_len)
        if B * Hkv * max_len > 1 << 36:                        # (refused: more rows than any card holds)
            assert step(B, Hq, Hkv, D, max_len) == -2 and need == 0
            continue
        assert step(B, Hq, Hkv, D, max_len) == -3, (B, Hq, Hkv, D, max_len)
        most = max(7 * B * Hq, 16384 * Hq // Hkv) * (4 * D + 8) + 256
        assert need <= most, (B, Hq, Hkv, D, max_len, need)
        assert need > 0 if max_len > 1024 else (need == 0 or max_len > 512), (B, Hq, Hkv, D, max_len, need)
    # 128 sequences of up to 131072 rows, 32/8 heads: 34 MB
    assert pkg.snapkv_decode_paged_workspace_bytes(128, 32, 8, 128, 131072) == 128 * 32 * 16 * (128 * 4 + 8)
