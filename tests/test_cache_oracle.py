"""The oracle of the 8-bit cache and the eviction against independent ground: torch's e4m3 type, brute force,
closed forms.  CPU only."""
import itertools
import math

import numpy as np
import pytest
import torch

from oracle import cache_oracle as co


def test_e4m3_rounding_is_torchs_over_a_dense_grid():
    grid = np.concatenate([np.linspace(-448, 448, 200001), np.ldexp(1.0, np.arange(-12, 9)),
                           np.ldexp(np.linspace(1, 2, 257), -7), np.ldexp(np.arange(0, 65) / 8.0, -9)])
    x = torch.from_numpy(grid.astype(np.float32))
    want = x.to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(co.e4m3_round(x.double().numpy()), want)
    assert np.isnan(co.e4m3_round(np.array([np.inf, -np.inf, np.nan]))).all()


@pytest.mark.parametrize("top", [0.0, 2.0 ** -133, 448 * 2.0 ** -126, 449 * 2.0 ** -126, 1.0, 447.9, 448.0, 448.1, 3.3895e38])
def test_block_scale_is_the_smallest_power_of_two_that_fits(top):
    s = co.block_scale(np.array([[top, -top / 3]]))
    assert top <= 448 * s and math.frexp(s)[0] == 0.5
    assert s == 2.0 ** -126 or top > 448 * (s / 2)


def test_quantising_again_changes_nothing_and_moving_scales_is_exact():
    rng = np.random.default_rng(0)
    x = rng.normal(size=(200, 32))
    codes, scales = co.quantise(x)
    v = co.values(codes, scales)
    again, scales2 = co.quantise(v)
    assert np.array_equal(co.values(again, scales2), v)
    # half a step of three fraction bits, or half the smallest step where the row is small beside its block
    assert (np.abs(v - x) <= np.maximum(np.abs(x) * 2.0 ** -4, np.repeat(scales, 64)[:200, None] * 2.0 ** -10)).all()


def test_appending_row_by_row_ends_with_the_scale_of_the_whole_block():
    rng = np.random.default_rng(1)
    x = rng.normal(size=(130, 16)) * np.exp2(rng.integers(-3, 4, size=(130, 1)))
    codes, scales = np.zeros((0, 16)), np.zeros(0)
    for row in x:
        codes, scales = co.append(codes, scales, row[None])
    want_codes, want_scales = co.quantise(x)
    assert np.array_equal(scales, want_scales)
    big = np.abs(want_codes) >= 2.0 ** -6                 # normal numbers: the rescaling was exact
    assert np.array_equal(codes[big], want_codes[big])


def test_attend_and_collected_small_by_hand():
    k = np.array([[0.0, 0.0], [2.0, 0.0]])
    v = np.array([[1.0, 0.0], [0.0, 1.0]])
    q = np.array([[[math.sqrt(2) * math.log(3) / 2, 7.0]]])
    out, lse, w = co.attend(q, k, v)
    assert np.allclose(out[0, 0], [0.25, 0.75]) and np.allclose(lse, math.log(4)) and np.allclose(w, [0.25, 0.75])
    out, lse, w = co.attend(np.ones((3, 1, 2)), k, v)     # three tokens, two rows: the first sees nothing
    assert np.array_equal(out[0, 0], [0, 0]) and lse[0, 0] == -np.inf and np.allclose(out[1, 0], v[0])
    assert np.isclose(w.sum(), 2.0)


def test_evict_against_brute_force():
    rng = np.random.default_rng(2)
    for n, keep, recent, sink in itertools.product([0, 1, 5, 9], [0, 1, 4, 20], [0, 2, 30], [0, 3]):
        acc = rng.integers(0, 4, size=n).astype(np.float32)
        got = co.evict(acc, keep, recent, sink)
        k = min(keep, n)
        assert got.sum() == k
        r = min(recent, k)
        s = min(sink, k - r)
        assert got[n - r:].all() and got[:s].all()
        mid = np.arange(s, n - r)
        best = max((tuple(sorted(c)) for c in itertools.combinations(mid, k - r - s)),
                   key=lambda c: (sum(acc[i] for i in c), tuple(-i for i in c)), default=())
        assert tuple(np.flatnonzero(got[s:n - r]) + s) == best
