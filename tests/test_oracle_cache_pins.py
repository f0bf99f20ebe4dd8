"""The cache's oracle against worked examples and independent arithmetic (CPU)."""
import math
from fractions import Fraction

import numpy as np
import pytest

from oracle import cache_ref as R


def test_codes_are_nearest_with_ties_to_the_even_code():
    # the largest magnitude 6 fixes the scale at 1 (byte 127); between neighbours of the grid the midpoints go to the even code
    x = np.zeros(32)
    x[:15] = [6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 0.26, 0.74, 1.26, 1.74, 2.51, 3.49, 5.01]
    code, byte = R.encode(x)
    assert byte.tolist() == [127]
    assert code[:15].tolist() == [7, 0, 2, 2, 4, 4, 6, 6, 1, 1, 3, 3, 5, 5, 7]
    code, _ = R.encode(-x)
    assert code[:15].tolist() == [15, 8, 10, 10, 12, 12, 14, 14, 9, 9, 11, 11, 13, 13, 15]


@pytest.mark.parametrize("top,byte", [(6.0, 127), (6.99, 127), (7.0, 128), (8.0, 128), (13.9, 128), (14.0, 129), (3.5, 127), (3.49, 126),
                                      (1.0, 126 - 1), (0.0, 1), (2.0 ** -140, 1), (3.0e38, 252), (2.0 ** 127, 252)])
def test_the_scale_is_the_least_that_keeps_the_largest_below_seven(top, byte):
    x = np.zeros(32)
    x[5] = -top
    assert R.encode(x)[1].tolist() == [byte]


def test_no_value_is_off_by_more_than_half_a_step_in_exact_arithmetic():
    rng = np.random.default_rng(0)
    grid = [Fraction(float(g)) for g in R.GRID]
    for _ in range(40):
        x = (rng.standard_normal(32) * 2.0 ** rng.integers(-20, 20)).astype(np.float32)
        code, byte = R.encode(x)
        scale = Fraction(2) ** (int(byte[0]) - 127)
        for a, c in zip(x, code):
            y = abs(Fraction(float(a))) / scale
            assert abs(y - grid[c & 7]) == min(abs(y - g) for g in grid)
            assert abs(y - grid[c & 7]) <= 1
            assert (c >= 8) == bool(np.signbit(a))


def test_decode_inverts_and_a_row_that_is_not_finite_reads_back_as_nan():
    x = np.random.default_rng(1).standard_normal((3, 64))
    values = R.decode(*R.encode(x))
    assert np.array_equal(R.decode(*R.encode(values)), values)
    k, v = x.copy(), x.copy()
    v[1, 40] = np.inf
    kk, vv = R.read_back(k, v)
    assert np.isnan(kk[1]).all() and np.isnan(vv[1]).all() and np.isfinite(kk[[0, 2]]).all() and np.isfinite(vv[[0, 2]]).all()


@pytest.mark.parametrize("D,P", [(64, 8), (128, 16), (256, 32)])
def test_places_cover_a_page_once(D, P):
    every = np.concatenate([np.concatenate(R.place(D, P, t)) for t in range(P)])
    assert np.array_equal(np.sort(every), np.arange(P * (D + D // 16)))
    # token 9 of head dimension 128: octet 1, place 1 of 8; channels 8 .. 15 are dword column 1
    if D == 128:
        key, value, ks, vs = R.place(D, P, 9)
        assert key[0] == 9 * 64 and value[4] == P * 64 + (16 + 1) * 32 + 4 and ks[2] == P * 128 + 38 and vs[2] == P * 132 + (4 + 2) * 8 + 1


def test_attention_by_hand():
    # two keys, scores 0 and ln 3: p = (1/4, 3/4)
    q = np.array([[1.0, 0.0]])
    k = np.array([[0.0, 5.0], [math.log(3.0), 1.0]])
    v = np.array([[4.0, 0.0], [0.0, -8.0]])
    out, lse, mass, worst = R.attention(q, k, v, np.ones((1, 2), bool), 1.0)
    assert np.allclose(out, [[1.0, -6.0]], atol=1e-15) and np.allclose(lse, math.log(4.0)) and np.allclose(mass, [[1.0, 6.0]])
    out, lse, _, _ = R.attention(q, k, v, np.zeros((1, 2), bool), 1.0)
    assert np.array_equal(out, np.zeros((1, 2))) and lse[0] == -np.inf
    k[0] = np.nan
    out, lse, _, _ = R.attention(np.repeat(q, 2, 0), k, v, np.array([[True, True], [False, True]]), 1.0)
    assert np.isnan(out[0]).all() and np.isnan(lse[0]) and np.array_equal(out[1], v[1])


def test_tree_and_words_by_hand():
    sees, good = R.tree_sees([-1, 0, 0, 1, 9], 4)
    assert good and sees.astype(int).tolist() == [[1, 0, 0, 0, 0], [1, 1, 0, 0, 0], [1, 0, 1, 0, 0], [1, 1, 0, 1, 0], [0] * 5]
    assert R.words_of(sees)[:, 0].tolist() == [1, 3, 5, 11, 0]
    sees, good = R.tree_sees([-1, 0, 2], 3)
    assert not good and sees.sum() == 1 and sees[0, 0]


def test_tables_by_hand():
    t = R.Tables(pages=8, sequences=4, width=3, P=8)
    assert t.reserve([0], [10]) == ([0], []) and t.table[0].tolist() == [0, 1, -1]
    t.lens[0] = 10
    assert t.fork([0, 0], [1, 2]) == [0, 0] and t.refs.tolist()[:2] == [3, 3]
    # three holders of page 1, all write: two copies, the last keeps it
    status, copied = t.reserve([0, 1, 2], [1, 7, 1])
    assert status == [0, 0, 0] and copied == [(1, 2), (1, 3)] and t.refs.tolist() == [3, 1, 1, 1, 1, 0, 0, 0]
    assert t.table.tolist() == [[0, 2, -1], [0, 3, 4], [0, 1, -1], [-1, -1, -1]]
    assert t.reserve([3, 0], [25, 15]) == ([2, 2], [])           # both wider than the table
    assert t.reserve([3], [24]) == ([0], []) and t.reserve([0, 2, 1], [14, 1, 1]) == ([1, 0, 0], [])
    # pages 5, 6, 7 are taken; a fork of sequence 2 shares page 1, and neither can be given a copy
    t.release([3])
    t.reserve([3], [24])
    t.lens[2] = 11
    t.release([1])
    assert t.fork([2], [1]) == [0] and t.refs.tolist() == [3, 2, 1, 0, 0, 1, 1, 1]
    t.refs[[3, 4]] = 1
    assert t.reserve([1, 2], [1, 1]) == ([1, 1], []) and t.refs[1] == 2
    t.refs[[3, 4]] = 0
    t.release([0, 1, 2, 3])
    assert not t.refs.any() and not t.held.any() and (t.table == -1).all()
