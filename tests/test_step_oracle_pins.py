"""Pins of the oracle for what surrounds attention in a step (no GPU needed)."""
import itertools

import numpy as np
import pytest

from oracle import paged_attention as orc
from oracle import paged_step as step


def _bits(x):
    return (np.asarray(x, np.float32).view(np.uint32) >> 16).astype(np.uint16)   # (cut, not rounded)


def _randn_bits(rng, *shape):
    return _bits(rng.standard_normal(shape))


def test_tables_by_hand():
    # 20 tokens behind 14 (2 of them fill the page there is, 16 a new one, 2 another); none behind 16; 1 behind 32
    tables, cu, pos, slots, nxt, cur, ok = step.step_tables([14, 16, 32], [20, 0, 1], [7, 3, 9, 4], [[5, -1, -1], [6, -1, -1], [1, 2, -1]], 23, 10)
    assert ok and cur == 3 and nxt == [34, 16, 33] and cu.tolist() == [0, 20, 20, 21]
    assert tables.tolist() == [[5, 7, 3], [6, -1, -1], [1, 2, 9]]
    assert pos.tolist() == list(range(14, 34)) + [32, 0, 0]
    assert slots.tolist() == [5 * 16 + 14, 5 * 16 + 15] + [7 * 16 + i for i in range(16)] + [3 * 16, 3 * 16 + 1, 9 * 16, -1, -1]


def test_tables_refuse_what_does_not_fit():
    free, tables = [7, 3, 9], [[5, -1], [6, -1], [4, -1], [1, -1]]
    *_, slots, nxt, cur, ok = step.step_tables([0, -1, 30, 3], [16, 1, 3, 2], free, tables, 40, 10)
    assert not ok and nxt == [16, -1, 30, 5] and cur == 1                       # the second has no length, the third no room in its row
    assert [s >= 0 for s in slots[:22]] == [True] * 16 + [False] * 4 + [True] * 2
    *_, nxt, cur, ok = step.step_tables([16, 16, 16, 3], [16, 16, 1, 2], free[:1], tables, 40, 10)
    assert not ok and nxt == [32, 16, 16, 5] and cur == 1                       # the list runs out; who needs no page goes on


@pytest.mark.parametrize("neighbours", [False, True])
def test_rotation(neighbours):
    rng = np.random.default_rng(1)
    x, y = rng.standard_normal((2, 5, 3, 64))
    inv = 10000.0 ** (-np.arange(24) / 24)
    turn = lambda v, p: step.rotate(v, np.broadcast_to(p, (1, 5)), inv, None, neighbours)
    assert np.allclose(np.linalg.norm(turn(x, 77), axis=-1), np.linalg.norm(x, axis=-1), rtol=1e-13)
    assert np.allclose(turn(turn(x, 30), 12), turn(x, 42), atol=1e-12)
    assert np.array_equal(turn(x, 9)[..., 48:], x[..., 48:]) and np.array_equal(turn(x, 0), x)
    dot = lambda a, b: np.sum(turn(x, a) * turn(y, b), -1)
    assert np.allclose(dot(100, 40), dot(161, 101), atol=1e-11)                  # only the distance counts


def test_rotation_axes_are_independent_rotations():
    rng = np.random.default_rng(2)
    x, pos, inv = rng.standard_normal((4, 2, 64)), rng.integers(0, 50, (3, 4)), rng.random(32)
    axis = np.arange(32) % 3
    y = step.rotate(x, pos, inv, axis)
    for a in range(3):                                                           # each axis alone, the others' frequencies at rest
        z = step.rotate(x, pos[a:a + 1], np.where(axis == a, inv, 0.0))
        j = np.where(axis == a)[0]
        assert np.array_equal(y[..., j], z[..., j]) and np.array_equal(y[..., j + 32], z[..., j + 32])


def test_score_is_a_bound_and_the_choice_is_the_best_subset():
    rng = np.random.default_rng(3)
    pool = orc.PagePool(9, 16, 2, 64)
    pool.k[:] = _randn_bits(rng, 9, 2, 16, 64)
    bounds = step.page_bounds(pool, np.arange(9 * 16), np.zeros((9, 2, 2, 64)))
    tables, q_bits = [rng.permutation(9)[:7].tolist()], _randn_bits(rng, 1, 8, 64)
    q, k = orc.widen(q_bits)[0], orc.widen(pool.k)
    for h in range(2):
        s = step.page_scores(q[4 * h:4 * h + 4], bounds[np.array(tables[0]), h])
        dots = np.einsum("gd,ptd->pgt", q[4 * h:4 * h + 4], k[np.array(tables[0]), h])
        assert np.all(s >= dots.max((1, 2)))
        lists, counts = step.select_pages(q_bits, bounds, tables, [7 * 16 - 5], 2, 4, 1, 1)
        best = max(itertools.combinations(range(1, 6), 2), key=lambda c: sum(s[list(c)]))
        assert lists[0, h].tolist() == [0, *best, 6] and counts[0, h] == 4


def test_choice_ties_and_what_is_not_a_number():
    bounds = np.ones((5, 1, 2, 64))
    q = _bits(np.ones((1, 1, 64)))
    pick = lambda: step.select_pages(q, bounds, [[0, 1, 2, 3, 4]], [80], 1, 2, 0, 0)[0][0, 0].tolist()
    assert pick() == [0, 1]
    bounds[3, 0, 1, 5] = np.nan
    assert pick() == [0, 3]
    bounds[2, 0, 1, 5] = np.inf
    assert pick() == [2, 3]


def test_attention_over_all_pages_is_attention():
    rng = np.random.default_rng(4)
    pool = orc.PagePool(8, 16, 2, 64)
    pool.k[:], pool.v[:] = _randn_bits(rng, 2, 8, 2, 16, 64)
    q = _randn_bits(rng, 2, 8, 64)
    tables, ctx = [[3, 1, 7, 0], [2, 6, -1, -1]], [55, 17]
    lists = np.array([[[2, 0, 3, 1]] * 2, [[0, 1, -1, -1]] * 2])
    o, l = step.decode_selected(pool, q, 8, tables, ctx, lists, [[4, 4], [2, 2]], 0.125)
    o2, l2 = orc.attn_decode(pool, q, 8, tables, ctx, 0.125)
    assert np.allclose(o, o2, atol=1e-14) and np.allclose(l, l2, atol=1e-14)
    o, l = step.decode_selected(pool, q, 8, tables, ctx, lists, [[0, 4], [2, 2]], 0.125)
    assert np.all(o[0, :4] == 0) and np.all(np.isneginf(l[0, :4])) and np.allclose(o[0, 4:], o2[0, 4:], atol=1e-14)
