"""The oracle of microscaled caches and shared prefixes pinned to tables, library conversions and the other oracle (no GPU needed)."""
import numpy as np
import pytest
import torch

from oracle import mx_oracle as orc
from oracle import serve_oracle

RNG = np.random.default_rng(5)


def test_element_values():
    e4m3 = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(orc.GRID["fp8"], e4m3) and orc.GRID["fp8"][-1] == 448
    assert list(orc.GRID["fp4"]) == [0, 0.5, 1, 1.5, 2, 3, 4, 6]
    for kind, n in (("fp8", 256), ("fp4", 16)):
        codes = np.arange(n).reshape(-1, 1).repeat(32, 1)
        got = orc.values(codes, np.full((n, 1), 130), kind)[:, 0]
        half = 8 * orc.GRID[kind]
        if kind == "fp8":
            half = np.append(half, np.nan)
        assert np.array_equal(got, np.concatenate([half, -half]), equal_nan=True)
    assert np.isnan(orc.values(np.zeros((1, 32)), [[255]], "fp4")).all()


def test_rounding_is_that_of_the_type():
    """Blocks whose largest value makes e zero: codes are torch's own conversion of the values."""
    x = RNG.standard_normal((400, 32)) * np.exp(3 * RNG.standard_normal((400, 1)))
    x = np.clip(x, -448, 448).astype(np.float32)
    x[:, 0] = 448
    codes, scales = orc.quantise(x, "fp8")
    assert (scales == 127).all()
    assert np.array_equal(codes, torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy())


@pytest.mark.parametrize("kind,most", [("fp8", 448.0), ("fp4", 6.0)])
def test_blocks_by_hand(kind, most):
    grid, top = orc.GRID[kind], len(orc.GRID[kind]) - 1
    one = lambda v: orc.quantise(np.pad([v], (0, 31)), kind)
    for v, byte in ((most, 127), (np.nextafter(most, 1e9), 128), (most / 2, 126), (2 * most, 128), (0.0, 10), (1e-300, 10)):
        assert one(v)[1] == [byte], v
    assert one(most)[0][0] == top and one(-most)[0][0] == top + (128 if kind == "fp8" else 8) and one(0.0)[0].sum() == 0
    row = np.zeros(32)
    row[0] = most
    row[1:5] = [(grid[1] + grid[2]) / 2, (grid[2] + grid[3]) / 2, -grid[1] / 2, np.nextafter(grid[1] / 2, 1)]
    sign = 128 if kind == "fp8" else 8
    assert list(orc.quantise(row, kind)[0][:5]) == [top, 2, 2, sign, 1]      # ties to the even code, signs of zero kept
    for bad in (np.inf, -np.inf, np.nan):
        x = np.ones((2, 64))
        x[1, 40] = bad
        codes, scales = orc.quantise(x, kind)
        assert scales[1, 1] == 255 and (codes[1, 32:] == 0).all() and (scales.reshape(-1)[:3] < 255).all()
        back = orc.values(codes, scales, kind)
        assert np.isnan(back[1, 32:]).all() and np.isfinite(back[0]).all() and np.isfinite(back[1, :32]).all()


@pytest.mark.parametrize("kind,step", [("fp8", 2.0 ** -4), ("fp4", 2.0 ** -2)])
def test_values_are_within_half_a_step(kind, step):
    x = RNG.standard_normal((50, 128)) * np.exp(8 * RNG.standard_normal((50, 1)))
    codes, scales = orc.quantise(x, kind)
    back = orc.values(codes, scales, kind)
    unit = np.repeat(np.ldexp(1.0, scales - 127), 32, axis=-1)
    low = orc.GRID[kind][1] / 2 * unit                                       # half a step of the smallest values
    assert (np.abs(back - x) <= np.maximum(step * np.abs(x), low)).all()
    again = orc.quantise(back, kind)
    assert np.array_equal(orc.values(*again, kind), back)
    assert np.array_equal(orc.unpack(orc.pack(codes, kind), kind), codes)


def test_shared_is_the_step_over_both_parts():
    B, Hq, Hkv, D, page = 5, 4, 2, 64, 4
    kp, vp = RNG.standard_normal((2, 30, page, Hkv, D))
    q = RNG.standard_normal((B, Hq, D))
    prefix_table, table = RNG.permutation(30)[:12].reshape(2, 6), RNG.integers(0, 30, (B, 3))
    prefix_lens, lens = [20, 8], [0, 5, 12, 3, 0]
    groups = [(0, 2), (2, 4)]
    out, lse, spread, reach = orc.decode_shared(q, kp, vp, prefix_table, prefix_lens, table, lens, groups)
    for b in range(4):
        whole = np.concatenate([prefix_table[b // 2, :prefix_lens[b // 2] // page], table[b]])[None]
        w = serve_oracle.decode_paged(q[b:b + 1], kp, vp, whole, [prefix_lens[b // 2] + lens[b]])
        for got, want in zip((out[b], lse[b], spread[b], reach[b]), w):
            assert np.allclose(got, want[0], rtol=1e-12)
    assert (out[4] == 0).all() and np.isneginf(lse[4]).all()                 # in no group, no rows of its own
