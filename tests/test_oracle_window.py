"""Pins of the windowed attention's reference."""

import numpy as np
import pytest

import oracle
from oracle import window


def _inputs(rng, B=3, G1=4, Hq=4, Hkv=2, D=64, cap=50):
    return (rng.normal(size=(B, G1, Hq, D)), rng.normal(size=(B, Hkv, cap, D)), rng.normal(size=(B, Hkv, cap, D)))


def test_no_window_is_the_verify_attention():
    rng = np.random.default_rng(0)
    q, k, v = _inputs(rng)
    kv_len, gamma = [50, 4, 30], [3, 3, 0]
    mask = (rng.random((3, 50)) < 0.7).astype(np.uint8)
    want, _ = oracle.verify_attention(q, k, v, kv_len, gamma, 0.2, mask)
    for w in (0, 50, 10 ** 6):
        got, _, st = window.verify_attention(q, k, v, kv_len, gamma, 0.2, mask, w, 0)
        np.testing.assert_allclose(got, want, rtol=1e-12, atol=1e-14)
        assert st == 0


@pytest.mark.parametrize("w,s", [(1, 0), (3, 0), (3, 2), (7, 20), (20, 1)])
def test_row_by_row_with_a_loop_over_keys(w, s):
    see = window.visible(23, 5, w, s)
    for i in range(6):
        pos = 17 + i
        for j in range(23):
            assert see[i, j] == (j <= pos and (pos - j < w or j < s))
    assert (see.sum(1) <= w + s).all()


def test_window_of_one_returns_the_row_itself():
    rng = np.random.default_rng(1)
    q, k, v = _inputs(rng)
    out, size, _ = window.verify_attention(q, k, v, [50, 30, 4], [3, 2, 3], 0.2, None, 1, 0)
    for b, (L, n) in enumerate(((50, 4), (30, 3), (4, 4))):
        want = np.repeat(v[b][:, L - n:L], 2, axis=0).swapaxes(0, 1)
        np.testing.assert_allclose(out[b, :n], want, rtol=1e-14)
        np.testing.assert_allclose(size[b, :n], np.abs(want), rtol=1e-14)
    assert (out[1, 3] == 0).all()


def test_unseen_entries_and_empty_rows():
    rng = np.random.default_rng(2)
    q, k, v = _inputs(rng, B=1)
    want, _, _ = window.verify_attention(q, k, v, [40], [2], 0.2, None, 8, 3)
    k[0, :, 3:30], v[0, :, 3:30], k[0, :, 40:], v[0, :, 40:] = np.nan, np.inf, np.nan, np.nan
    got, _, _ = window.verify_attention(q, k, v, [40], [2], 0.2, None, 8, 3)
    np.testing.assert_array_equal(got, want)
    mask = np.ones((1, 50), np.uint8)
    mask[0, 30:] = 0
    out, _, _ = window.verify_attention(q, k, v, [40], [2], 0.2, mask, 8, 0)
    assert (out == 0).all()
