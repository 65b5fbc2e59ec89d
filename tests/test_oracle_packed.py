"""Pins of the packed-sequence oracle: closed forms and invariants."""

import numpy as np
import pytest

from oracle import packed as P


def test_rotation_by_a_quarter_turn():
    x = np.arange(1.0, 5.0).reshape(1, 1, 4)
    quarter = [np.pi / 2, np.pi / 2]
    assert np.allclose(P.rotate(x, np.array([[1]]), quarter, [4], P.PAIRS), [[[-2, 1, -4, 3]]])
    assert np.allclose(P.rotate(x, np.array([[1]]), quarter, [4], P.HALVES), [[[-3, -4, 1, 2]]])
    # two axes: the second pair turns with the second position
    assert np.allclose(P.rotate(x, np.array([[0, 1]]), quarter, [2, 2], P.PAIRS), [[[1, 2, -4, 3]]])


@pytest.mark.parametrize("pairing", [P.PAIRS, P.HALVES])
def test_products_depend_on_the_distance_alone(pairing):
    rng = np.random.default_rng(0)
    q, k = rng.normal(size=(2, 1, 1, 16))
    f = rng.uniform(0.01, 1, 6)
    dot = [np.vdot(P.rotate(q, np.array([[a, 3 * a]]), f, [4, 8], pairing), P.rotate(k, np.array([[a + 5, 3 * a - 2]]), f, [4, 8], pairing))
           for a in (0, 7, 100000)]
    assert np.allclose(dot, dot[0])
    y = P.rotate(q, np.array([[9, 4]]), f, [4, 8], pairing)
    assert np.allclose(P.rotate(y, np.array([[-9, -4]]), f, [4, 8], pairing), q)
    assert np.array_equal(y[..., 12:], q[..., 12:])


def test_far_positions_keep_their_angle():
    # 2 pi / 1000 radians a position: position 2^31 - 648 turns as its remainder modulo 1000
    f = [2 * np.pi / 1000]
    x = np.array([[[1.0, 0.0]]])
    far = 2 ** 31 - 648
    assert np.allclose(P.rotate(x, np.array([[far]]), f, [2], P.PAIRS), P.rotate(x, np.array([[far % 1000]]), f, [2], P.PAIRS), atol=1e-9)


def test_norm_has_mean_square_one():
    x = np.random.default_rng(1).normal(size=(3, 2, 8)) * 7
    y = P.rms_norm(x, np.ones(8), 0.0)
    assert np.allclose((y * y).mean(-1), 1)
    assert np.allclose(P.rms_norm(x, 2 * np.ones(8), 0.0), 2 * y)


def test_attention_of_equal_scores_is_the_mean_of_what_is_seen():
    rng = np.random.default_rng(2)
    v = rng.normal(size=(5, 1, 4))
    o, _ = P.attention(np.zeros((3, 2, 4)), rng.normal(size=(5, 1, 4)), v, True, 1.0)
    for i in range(3):
        for h in range(2):
            assert np.allclose(o[i, h], v[:3 + i, 0].mean(0))
    # more new rows than keys: the first rows see nothing
    o, _ = P.attention(np.zeros((4, 1, 4)), v[:2], v[:2], True, 1.0)
    assert not o[:2].any() and np.allclose(o[2, 0], v[0, 0]) and np.allclose(o[3, 0], v[:2, 0].mean(0))


def test_attention_weights_follow_the_scores():
    q, k = np.array([[[1.0, 0]]]), np.array([[[np.log(3), 0]], [[0.0, 5]]])
    o, a = P.attention(q, k, np.array([[[1.0, 0]], [[0.0, -1]]]), False, 1.0)
    assert np.allclose(o, [[[0.75, -0.25]]]) and np.allclose(a, [[[0.75, 0.25]]])
