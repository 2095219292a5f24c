"""Pins of the learned-policy checker: hand-worked values, limits and differences (CPU)."""
from __future__ import annotations

import math

import numpy as np
import pytest

from oracle import policy as P

INF = math.inf


def test_distill_by_hand():
    # p = (1/2, 1/4, 1/4), q = (1/3, 2/3) on hosts 0 and 2
    x = np.log(np.array([[2.0, 1.0, 1.0]]))
    loss, grad = P.distill(x, np.array([[0, 2]]), np.log(np.array([[1.0, 2.0]])))
    want = (1 / 3) * math.log((1 / 3) / (1 / 2)) + (2 / 3) * math.log((2 / 3) / (1 / 4))
    np.testing.assert_allclose(loss, [want], rtol=1e-14)
    np.testing.assert_allclose(grad, [[1 / 2 - 1 / 3, 1 / 4, 1 / 4 - 2 / 3]], rtol=1e-14)


def test_distill_entries_that_do_not_count():
    x = np.array([[0.0, -INF, 1.0, 2.0]])
    full = P.distill(x, np.array([[3, 2]]), np.array([[0.5, 0.25]]))
    for hosts, t in (([[3, 2, -1, 4, 1]], [[0.5, 0.25, 9.0, 9.0, 9.0]]), ([[3, 0, 2]], [[0.5, -INF, 0.25]])):
        got = P.distill(x, np.array(hosts), np.array(t))
        np.testing.assert_allclose(got[0], full[0], rtol=1e-14)
        np.testing.assert_allclose(got[1], full[1], rtol=1e-14)
    for x0, hosts in ((x, [[-1, 1]]), (np.full((1, 4), -INF), [[0, 1]])):
        loss, grad = P.distill(x0, np.array(hosts), np.zeros((1, 2)))
        assert loss[0] == 0 and not grad.any()


def test_distill_equal_policies_have_no_loss():
    x = np.array([[0.3, -1.0, 0.7]])
    loss, grad = P.distill(x, np.array([[0, 1, 2]]), x, temperature=1.7)
    np.testing.assert_allclose(loss, 0, atol=1e-14)
    np.testing.assert_allclose(grad, 0, atol=1e-14)


@pytest.mark.parametrize("temperature", [0.5, 1.0, 2.5])
def test_distill_gradient_is_the_slope(temperature):
    rng = np.random.default_rng(1)
    x, hosts, t = rng.normal(size=(3, 7)), np.array([[0, 3, 3], [6, -1, 2], [1, 5, 4]]), rng.normal(size=(3, 3))
    x[0, 5] = -INF
    _, grad = P.distill(x, hosts, t, temperature)
    h = 1e-5
    for j in range(7):
        up, down = x.copy(), x.copy()
        up[:, j] += h
        down[:, j] -= h
        slope = (P.distill(up, hosts, t, temperature)[0] - P.distill(down, hosts, t, temperature)[0]) / (2 * h)
        np.testing.assert_allclose(grad[:, j], slope, atol=1e-8)


def test_balance_by_hand():
    # two rows, f = (3/4, 1/4), p = (1/2, 1/2) and (1/4, 3/4); a third row without a choice is left out
    x = np.log(np.array([[1.0, 1.0], [1.0, 3.0], [5.0, 1.0]]))
    loss, counts, shares, grad = P.balance(x, np.array([[0, 0], [1, 0], [-1, 2]]))
    assert counts.tolist() == [3, 1]
    np.testing.assert_allclose(shares, [3 / 8, 5 / 8], rtol=1e-14)
    np.testing.assert_allclose(loss, 2 * (3 / 4 * 3 / 8 + 1 / 4 * 5 / 8), rtol=1e-14)
    np.testing.assert_allclose(grad, [[1 / 2 * (3 / 4 - 1 / 2), 1 / 2 * (1 / 4 - 1 / 2)],
                                      [1 / 4 * (3 / 4 - 3 / 8), 3 / 4 * (1 / 4 - 3 / 8)], [0, 0]], rtol=1e-13)


def test_balance_is_one_when_even_and_zero_when_empty():
    loss, _, shares, _ = P.balance(np.zeros((4, 4)), np.array([[0], [1], [1], [1]]))
    np.testing.assert_allclose(loss, 1.0)
    np.testing.assert_allclose(shares, 0.25)
    loss, counts, shares, grad = P.balance(np.zeros((4, 4)), np.full((4, 2), -1))
    assert loss == 0 and not counts.any() and not shares.any() and not grad.any()


def test_balance_gradient_is_the_slope():
    rng = np.random.default_rng(2)
    x, hosts = rng.normal(size=(4, 5)), np.array([[0, 1], [0, 4], [-1, -1], [0, 2]])
    x[0, 3] = -INF
    grad = P.balance(x, hosts)[3]
    h = 1e-5
    for r in range(4):
        for j in range(5):
            up, down = x.copy(), x.copy()
            up[r, j] += h
            down[r, j] -= h
            np.testing.assert_allclose(grad[r, j], (P.balance(up, hosts)[0] - P.balance(down, hosts)[0]) / (2 * h), atol=1e-9)


T_ONE = np.float32(1.4426950408889634)   # c = 1: whole logits have exact weights


def test_sample_weights_by_hand():
    _, w = P.sample_weights([3.0, 2.0, -INF, math.nan, 1.0, -40.0], T_ONE)
    assert w == [2 ** 31, 2 ** 30, 0, 0, 2 ** 29, 0]


def test_sample_filters_by_hand():
    x = [1.0, 3.0, 2.0, 3.0, 2.0]   # weights 1/4, 1, 1/2, 1, 1/2 of 2^31
    one = 2 ** 31
    assert P.sample_kept(x, T_ONE, top_k=3) == [0, one, one // 2, one, 0]          # tie at 2.0: the lower index
    assert P.sample_kept(x, T_ONE, top_p=0.5) == [0, one, 0, one, 0]               # 1.625 of 3.25
    assert P.sample_kept(x, T_ONE, top_k=4, top_p=0.75) == [0, one, one // 2, one, 0]   # 2.25 of 3.0
    assert P.sample_kept(x, T_ONE, min_p=0.5) == [0, one, one // 2, one, one // 2]
    assert P.sample_kept(x, 0.0) == [0, one, 0, 0, 0]
    assert P.sample_kept(x, T_ONE, top_p=0.0) == [0, one, 0, 0, 0]


def test_draws_are_distinct_and_in_index_order():
    w = [1, 0, 2, 1]
    assert P.draw(w, [0.0, 0.0, 0.0, 0.0]) == ([0, 2, 3, -1], 3)
    assert P.draw(w, [0.25, 0.5]) == ([2, 3], 2)       # t = 1 of 4 -> host 2; t = 1 of 2 -> host 3
    assert P.draw(w, [1.0, -1.0, math.nan]) == ([3, 0, 2], 3)
    assert P.draw([0, 0], [0.5]) == ([-1], 0)
