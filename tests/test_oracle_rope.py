"""Pins of the norm-and-rotation reference: closed forms and invariants."""

import numpy as np
import pytest

from oracle import rope


def _table(n, rot, theta=10000.0):
    a = np.arange(n)[:, None] * theta ** (-np.arange(0, rot, 2) / rot)
    return np.concatenate([np.cos(a), np.sin(a)], -1)


@pytest.mark.parametrize("interleaved", [False, True])
def test_scores_depend_on_the_distance_alone(interleaved):
    rng = np.random.default_rng(1)
    D, n = 64, 40
    t = _table(n, D)
    q, k = rng.normal(size=D), rng.normal(size=D)
    for d in (0, 3, 11):
        dots = []
        for p in (0, 5, 20):
            a = rope.turn(q, t[p + d, :32], t[p + d, 32:], interleaved)
            c = rope.turn(k, t[p, :32], t[p, 32:], interleaved)
            dots.append(a @ c)
        np.testing.assert_allclose(dots, dots[0], rtol=1e-12, atol=1e-12)


def test_pairs_turn_as_complex_numbers_and_the_rest_stays():
    rng = np.random.default_rng(2)
    x = rng.normal(size=(3, 64))
    a = rng.normal(size=16)
    y = rope.turn(x, np.cos(a), np.sin(a), False)
    z = (x[:, :16] + 1j * x[:, 16:32]) * np.exp(1j * a)
    np.testing.assert_allclose(y[:, :16], z.real, rtol=1e-14, atol=1e-14)
    np.testing.assert_allclose(y[:, 16:32], z.imag, rtol=1e-14, atol=1e-14)
    np.testing.assert_array_equal(y[:, 32:], x[:, 32:])
    y = rope.turn(x, np.cos(a), np.sin(a), True)
    z = (x[:, 0:32:2] + 1j * x[:, 1:32:2]) * np.exp(1j * a)
    np.testing.assert_allclose(y[:, 0:32:2], z.real, rtol=1e-14, atol=1e-14)
    np.testing.assert_allclose(y[:, 1:32:2], z.imag, rtol=1e-14, atol=1e-14)


def test_normed_head_has_the_weight_as_its_root_mean_square():
    rng = np.random.default_rng(3)
    x = rng.normal(size=(5, 128)) * 37.0
    y = rope.norm_head(x, np.full(128, 3.0), 0.0)
    np.testing.assert_allclose(np.sqrt((y ** 2).mean(-1)), 3.0, rtol=1e-12)
    assert rope.norm_head(x, None, 1e-6) is x


def test_bad_data_is_flagged_and_not_an_output():
    t = _table(10, 16)
    x = np.ones((4, 3, 1, 64))
    y, live, _, st = rope.norm_rope(x, None, 1e-6, t, [0, 8, -1, 0], [2, 2, 0, 3])
    assert st == rope.ST_GAMMA | rope.ST_POSITION
    assert live.tolist() == [[True] * 3, [False] * 3, [False] * 3, [False] * 3]
    _, live, _, st = rope.norm_rope(x, None, 1e-6, t, [7, 9, 0, 1], [2, 0, 0, 1])  # the table's last positions
    assert st == 0 and live.sum() == 3 + 1 + 1 + 2
