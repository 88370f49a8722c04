"""The largest calls around pages that a launch holds: one token more is refused before it (no GPU needed: the pointers are made up, and `starts` at an odd
address is refused behind the sizes)."""
import pytest

import paper_2404_14469_amd as pkg

FAKE, ODD = 0x1000, 0x1002
MOST = (1 << 26) - 4


def append(T, cache):
    L = pkg.load()
    rows = (T, 1, 0, 1, 64, 0, 0, 64, 0, 64, 0, None, None, 0, 0, 0)
    if cache is None:
        return L.snapkv_append_paged(0, None, FAKE, FAKE, FAKE, ODD, None, *rows, FAKE, FAKE, FAKE, 1, 1, 16, None, 0, 0, None, 0, 0, None)
    return L.snapkv_append_paged_mx(0, cache, None, FAKE, FAKE, FAKE, ODD, None, *rows, FAKE, FAKE, FAKE, FAKE, FAKE, 1, 1, 16, None, 0, 0, None, 0, 0, None)


def read(T):
    return pkg.load().snapkv_read_paged_mx(0, 1, FAKE, FAKE, FAKE, FAKE, FAKE, 1, 1, 16, FAKE, ODD, T, 1, 1, 64, FAKE, 64, 0, FAKE, 64, 0, None)


@pytest.mark.parametrize("call", [lambda T: append(T, None), lambda T: append(T, 1), lambda T: append(T, 2), read])
def test_tokens_of_a_call(call):
    assert [call(T) for T in (MOST - 1, MOST)] == [-3, -3]
    assert [call(MOST + i) for i in range(1, 6)] == [-2] * 5
