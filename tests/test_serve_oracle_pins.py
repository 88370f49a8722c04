"""Pins of oracle/serve_oracle.py: closed forms, invariants and library routines (CPU only)."""
import numpy as np
import pytest
import scipy.special

from oracle import serve_oracle as orc


def angles(P, half, rng=None):
    a = np.arange(P)[:, None] * (10000.0 ** (-np.arange(half) / half))[None]
    return np.cos(a), np.sin(a)


def test_position_zero_and_a_quarter_turn():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((2, 3, 8))
    cos, sin = angles(4, 4)
    assert np.array_equal(orc.rotate(x, [0, 0], cos, sin, False), x)
    quarter = orc.rotate(x, [0, 0], np.zeros((1, 4)), np.ones((1, 4)), False)
    assert np.array_equal(quarter[..., :4], -x[..., 4:]) and np.array_equal(quarter[..., 4:], x[..., :4])
    part = orc.rotate(x, [3, 1], cos[:, :2], sin[:, :2], True)
    assert np.array_equal(part[..., 4:], x[..., 4:]) and not np.array_equal(part[..., :4], x[..., :4])
    assert np.array_equal(orc.rotate(x, [-5, 99], cos, sin, False), orc.rotate(x, [0, 3], cos, sin, False))   # clamped


@pytest.mark.parametrize("interleaved", [False, True])
def test_turns_add_and_dot_products_see_differences(interleaved):
    rng = np.random.default_rng(2)
    x, y = rng.standard_normal((2, 1, 1, 16))
    cos, sin = angles(64, 8)
    at = lambda z, p: orc.rotate(z, [p], cos, sin, interleaved)
    assert np.allclose(at(at(x, 5), 7), at(x, 12), atol=1e-12)
    assert np.isclose((at(x, 40) * at(y, 33)).sum(), (at(x, 9) * at(y, 2)).sum(), atol=1e-12)
    assert np.isclose((at(x, 11) ** 2).sum(), (x ** 2).sum())


def test_interleaved_pairs_are_a_permutation_of_the_halves():
    rng = np.random.default_rng(3)
    x = rng.standard_normal((3, 2, 16))
    cos, sin = angles(10, 8)
    perm = np.arange(16).reshape(2, 8).T.reshape(-1)       # 0 8 1 9 ...
    assert np.allclose(orc.rotate(x[..., perm], [1, 4, 9], cos, sin, True), orc.rotate(x, [1, 4, 9], cos, sin, False)[..., perm])


def test_append_is_plain_indexing_and_skips_what_has_no_page():
    rng = np.random.default_rng(4)
    pages = rng.standard_normal((6, 4, 2, 3))
    k = rng.standard_normal((9, 2, 3))
    table = np.array([[5, 0, 2], [1, -1, 9]])
    got, same = orc.append(pages, pages, k, k, table, [3, 2], [0, 5, 8])
    assert np.array_equal(got, same)
    want = pages.copy()
    want[5, 3], want[0, 0], want[0, 1], want[0, 2], want[0, 3] = k[0], k[1], k[2], k[3], k[4]
    want[1, 2], want[1, 3] = k[5], k[6]                     # the third token's page is -1; token 8 is behind the last sequence
    assert np.array_equal(got, want)


def test_prompt_closed_forms_and_scipy():
    rng = np.random.default_rng(5)
    q, k, v = rng.standard_normal((7, 4, 8)), rng.standard_normal((7, 2, 8)), rng.standard_normal((7, 2, 8))
    cu = [0, 1, 1, 6]                                       # one token, an empty prompt, five, one behind the last
    out, lse, spread, reach = orc.prompt_attention(q, k, v, cu)
    assert np.allclose(out[0], np.repeat(v[0], 2, axis=0)) and np.isnan(out[6]).all() and np.isnan(lse[:, 6]).all()
    s = q[3, 3] @ k[1:4, 1].T / np.sqrt(8.0)                # token 2 of the third prompt, head 3
    assert np.allclose(out[3, 3], scipy.special.softmax(s) @ v[1:4, 1]) and np.isclose(lse[3, 3], scipy.special.logsumexp(s))
    flat, flat_lse, mean_abs, _ = orc.prompt_attention(np.zeros_like(q), k, v, cu)
    for i in range(1, 6):
        assert np.allclose(flat[i, 0], v[1:i + 1, 0].mean(axis=0)) and np.isclose(flat_lse[0, i], np.log(i))
        assert np.allclose(mean_abs[i, 2], np.abs(v[1:i + 1, 1]).mean(axis=0))
    assert (reach[:, :6] >= np.abs(lse[:, :6]) - np.log(5) - 1e-9).all() and (spread[:6] >= np.abs(out[:6]) - 1e-12).all()


def test_a_prompts_last_row_is_the_step_over_its_pages():
    rng = np.random.default_rng(6)
    q, k, v = rng.standard_normal((11, 4, 8)), rng.standard_normal((11, 2, 8)), rng.standard_normal((11, 2, 8))
    table = np.array([[2, 3, 0], [1, 7, 7]])
    pool = np.full((4, 4, 2, 8), np.nan)
    kp, vp = orc.append(pool, pool, k, v, table, [0, 0], [0, 9, 11])
    out, lse, spread, reach = orc.prompt_attention(q, k, v, [0, 9, 11])
    got = orc.decode_paged(q[[8, 10]], kp, vp, table, [9, 2])
    for a, b in zip(got, (out[[8, 10]], lse[:, [8, 10]].T, spread[[8, 10]], reach[:, [8, 10]].T)):
        assert np.allclose(a, b)
    none = orc.decode_paged(q[:2], kp, vp, table, [0, 1])
    assert (none[0][0] == 0).all() and np.isneginf(none[1][0]).all() and np.allclose(none[0][1, 0], v[9, 0])
