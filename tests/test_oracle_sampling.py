"""Pins of the oracle for moved keys, rules on logits and drawn tokens: closed forms, hand-worked rows, brute force."""
import math

import numpy as np
import pytest
import torch

from oracle import actkv_oracle as O


def test_turns_add():
    g = np.random.default_rng(1)
    k, freq = g.normal(size=(7, 12)), np.array([1.0, 0.3, 0.01, 0.5])
    p, q = g.integers(0, 1000, (2, 2, 7))
    at = lambda pos: O.rotate(k[:, None], pos, freq, [1, 3], True)[:, 0]
    np.testing.assert_allclose(O.reposition_unit(at(p), p, q, freq, freq, [1, 3], True), at(q), atol=1e-9)
    slow = lambda pos: O.rotate(k[:, None], pos, freq / 4, [1, 3], True)[:, 0]
    np.testing.assert_allclose(O.reposition_unit(at(p), p, p, freq, freq / 4, [1, 3], True), slow(p), atol=1e-9)


def test_a_quarter_turn_by_hand():
    y = O.turn(np.array([[1.0, 2.0, 3.0, 4.0, 9.0]]), np.array([[math.pi / 2, 0.0]]), False)
    np.testing.assert_allclose(y, [[-3.0, 2.0, 1.0, 4.0, 9.0]], atol=1e-12)
    y = O.turn(np.array([[1.0, 2.0, 3.0, 4.0, 9.0]]), np.array([[math.pi / 2, math.pi]]), True)
    np.testing.assert_allclose(y, [[-2.0, 1.0, -3.0, -4.0, 9.0]], atol=1e-12)


def test_dot_products_depend_on_distances_only():
    g = np.random.default_rng(2)
    q, k, freq = g.normal(size=(1, 8)), g.normal(size=(1, 8)), np.array([1.0, 0.2, 0.03, 0.7])
    turn = lambda x, p: O.turn(x, np.array([[p]]) * freq, False)
    a = (turn(q, 90) @ turn(k, 71).T).item()
    moved = O.reposition_unit(turn(k, 71), [[71]], [[5]], freq, freq, [4], False)
    np.testing.assert_allclose((turn(q, 24) @ moved.T).item(), a)


def test_a_penalized_row_by_hand():
    z = [2.0, -2.0, 1.0, 4.0, 0.5]
    out = O.penalize_row(z, [0, 1, 3, 3, 9, -1], 2, 2.0, 0.25, 0.5, {4: 1.5, 3: -1.0}, np.array([1, 1, 0, 1, 1], dtype=bool))
    # 0 and 1 in the prompt: only repetition; 3 generated twice: (4 - 1) / 2 - 0.5 - 0.5; 4 only biased; 2 masked
    np.testing.assert_allclose(out, [1.0, -4.0, -np.inf, 0.5, 2.0])


def test_no_rules_change_nothing():
    z = np.random.default_rng(0).normal(size=20)
    np.testing.assert_array_equal(O.penalize_row(z, [3, 4, 4], 1, 1.0, 0.0, 0.0, {}, None), z)


def test_drawn_rows_by_hand():
    z = np.log(np.array([0.1, 0.4, 0.2, 0.3]))
    draw = lambda u, k=0, p=1.0, m=0.0, t=1.0: O.sample_row(z, u, t, k, p, m)
    assert [draw(u)[0] for u in (0.0, 0.05, 0.15, 0.49, 0.51, 0.69, 0.71, 1.0)] == [0, 0, 1, 1, 2, 2, 3, 3]
    assert draw(0.2)[2] == 4 and math.isclose(draw(0.2)[1], math.log(0.4))
    assert draw(0.9, k=2) == (3, pytest.approx(math.log(0.3 / 0.7)), 2) and draw(0.0, k=2)[0] == 1
    assert draw(0.0, p=0.65)[2] == 2 and draw(0.0, p=0.75)[2] == 3 and draw(0.0, p=0.3)[2] == 1
    assert draw(0.0, m=0.6)[2] == 2 and draw(0.0, m=2.0)[2] == 1
    assert draw(0.99, t=0.0) == (1, 0.0, 1)
    assert O.sample_row(np.array([1.0, 1.0, 1.0]), 0.99, 1.0, 2, 1.0, 0.0)[::2] == (1, 2)        # equal ones: the lower token first
    assert O.sample_row(np.full(3, -np.inf), 0.5, 1.0, 0, 1.0, 0.0) == (-1, -np.inf, 0)
    assert O.sample_row(np.array([0.0, np.nan]), 0.5, 1.0, 0, 1.0, 0.0)[0] == -1


def test_draws_follow_the_softmax():
    z = np.random.default_rng(3).normal(size=9) * 2
    p = torch.softmax(torch.from_numpy(z) / 0.7, 0).numpy()
    u = (np.arange(20000) + 0.5) / 20000
    got = np.bincount([O.sample_row(z, x, 0.7, 0, 1.0, 0.0)[0] for x in u], minlength=9) / 20000
    assert np.abs(got - p).max() <= 1e-4                         # evenly spaced numbers: off by less than two of them
