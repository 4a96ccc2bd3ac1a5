"""Pins of the serving oracle: hand values, special cases and brute force (CPU)."""
import math

import numpy as np

from oracle import cache_oracle as O


def test_what_a_row_sees():
    assert O.sees(5, 1, 1) == [5]
    assert O.sees(5, 3, 3) == [3, 4, 5]
    assert O.sees(5, 2, 4) == [4, 5, 0, 0]
    assert O.sees(1, 3, 3) == [0, 0, 1]
    assert O.sees(0, 2, 2) == [0, 0]
    assert O.sees(4, 0, 2) == [0, 0]


def test_attend_by_hand():
    k = np.array([[0.0], [math.log(3.0)]])
    v = np.array([[4.0], [8.0]])
    there = np.array([True, True])
    out, lse, p = O.attend(np.array([1.0]), k, v, 2, there, 1.0, 0.0)
    assert np.allclose(p, [0.25, 0.75]) and np.allclose(out, 7.0) and np.isclose(lse, math.log(4.0))
    out, lse, p = O.attend(np.array([1.0]), k, v, 1, there, 1.0, 0.0)
    assert np.allclose(p, [1.0, 0.0]) and np.allclose(out, 4.0) and lse == 0.0
    out, lse, p = O.attend(np.array([1.0]), k, v, 0, there, 1.0, 0.0)
    assert lse == -np.inf and not out.any() and not p.any()
    # the page of the first slot is not there; what it holds is not looked at
    out, lse, p = O.attend(np.array([1.0]), np.array([[np.nan], [1.0]]), np.array([[np.inf], [8.0]]), 2, np.array([False, True]), 1.0, 0.0)
    assert np.allclose(p, [0.0, 1.0]) and np.allclose(out, 8.0) and lse == 1.0
    # a cap of 2 holds logits below 2: weights of 1e9 and -1e9 are those of 2 and -2
    out, lse, p = O.attend(np.array([1.0]), np.array([[1e9], [-1e9]]), v, 2, there, 1.0, 2.0)
    assert np.isclose(p[0], 1 / (1 + math.exp(-4.0)))


def test_append():
    assert O.append(3, 10, 2, 8) == ([(0, 3, 10), (1, 4, 11)], 5, 12)
    assert O.append(7, 10, 3, 8) == ([(0, 7, 10)], 8, 13)
    assert O.append(8, 0, 1, 8) == ([], 8, 1)


def test_what_stays():
    there = [True] * 6
    mass = [0.5, 2.0, float("nan"), 2.0, -math.inf, 0.1]
    keys = O.rank_keys(mass, [5, 6, 7, 8, 9, 3], there, 10, 0, 0)
    assert O.evict_keep([keys], 6) == [[0, 1, 2, 3, 4, 5]]
    assert O.evict_keep([keys], 5) == [[0, 1, 3, 4, 5]]          # NaN goes first, behind -inf
    assert O.evict_keep([keys], 4) == [[0, 1, 3, 5]]
    assert O.evict_keep([keys], 1) == [[1]]                      # equal mass: the lower slot
    assert O.evict_keep([keys], 0) == [[]]
    keys = O.rank_keys(mass, [5, 6, 7, 8, 9, 3], there, 10, 4, 1)      # positions 3 and 9 are protected
    assert O.evict_keep([keys], 3) == [[1, 4, 5]]
    assert O.evict_keep([keys], 1) == [[4]]                      # the budget does not hold both
    keys = O.rank_keys(mass, [5, 6, 7, 8, 9, 3], [True, False] * 3, 10, 0, 0)
    assert O.evict_keep([keys], 2) == [[0, 4]]
    # a pool: equal mass stays in the lower head
    a, b = [(2, 1.0), (2, 3.0)], [(2, 3.0), (2, 2.0)]
    assert O.evict_keep([a, b], 2) == [[1], [0]]
    assert O.evict_keep([a, b], 1) == [[1], []]


def test_a_page_that_is_not_there_goes_before_a_weight_that_is_no_number():
    mass = [float("nan"), 2.0, float("nan"), 2.0, -math.inf, 0.1]
    keys = O.rank_keys(mass, [5, 6, 7, 8, 9, 3], [True, False, True, False, True, True], 10, 0, 0)
    assert O.evict_keep([keys], 5) == [[0, 1, 2, 4, 5]]
    assert O.evict_keep([keys], 4) == [[0, 2, 4, 5]]
    assert O.evict_keep([keys], 3) == [[0, 4, 5]]
    assert O.evict_keep([keys], 1) == [[5]]


def test_moves():
    assert O.evict_moves([0, 1, 2], 5) == []
    assert O.evict_moves([2, 3, 4], 5) == [(0, 3), (1, 4)]
    assert O.evict_moves([0, 4], 6) == [(1, 4)]
    assert O.evict_moves([], 6) == []
    rng = np.random.default_rng(2)
    for _ in range(200):
        c = int(rng.integers(1, 40))
        stay = sorted(rng.permutation(c)[:int(rng.integers(0, c + 1))].tolist())
        moves = O.evict_moves(stay, c)
        slots = list(range(c))
        for to, frm in moves:
            assert to < len(stay) <= frm and to not in stay and frm in stay
            slots[to] = frm
        assert sorted(slots[:len(stay)]) == stay and len(moves) == sum(s >= len(stay) for s in stay)
