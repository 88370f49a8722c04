"""Outputs whose rows overlap are refused (no GPU needed: what is taken is called without tokens, or refused by a later check)."""
import pytest

import paper_2404_14469_amd as pkg

FAKE, ODD = 0x1000, 0x1002      # never dereferenced: validation comes first


def append(Hq, Hkv, qor, qoh, kor, koh, T=100):
    return pkg.load().snapkv_append_paged(0, FAKE, FAKE, FAKE, FAKE, FAKE, ODD, T, 3, Hq, Hkv, 64, Hq * 64, 64, Hkv * 64, 64, Hkv * 64, 0, FAKE,
                                          FAKE, 4096, 64, 0, FAKE, FAKE, FAKE, 10, 30, 16, FAKE, qor, qoh, FAKE, kor, koh, None)


@pytest.mark.parametrize("kw,code", [
    (dict(qor=512, qoh=0), -1), (dict(qor=512, qoh=56), -1), (dict(kor=128, koh=0), -1), (dict(kor=128, koh=32), -1),     # heads meet
    (dict(qor=448, qoh=64), -1), (dict(kor=64, koh=64), -1), (dict(qor=64, qoh=64), -1), (dict(qor=64, qoh=64 * 99), -1),   # tokens and heads meet
    (dict(qor=512, qoh=64), -3), (dict(qor=64, qoh=6400), -3), (dict(qor=800, qoh=72), -3), (dict(kor=64, koh=6400), -3),   # (the odd address)
    (dict(Hq=1, Hkv=1, qor=64, qoh=0, kor=64, koh=0), -3),                             # a stride of one head does not matter
    (dict(T=1, qor=64, qoh=64), -3),                                                   # nor that of one token
])
def test_append_refuses_outputs_that_overlap(kw, code):
    a = dict(Hq=8, Hkv=2, qor=512, qoh=64, kor=128, koh=64)
    a.update(kw)
    assert append(**a) == code
