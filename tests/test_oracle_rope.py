"""Pins of the rotary oracle (CPU): hand-worked positions, the rotation's properties, finite differences."""
import numpy as np
import pytest

from oracle import rope as orope
from oracle import segments as oseg


def test_positions_by_hand():
    # two steps: a 2x3 screenshot with 2 text tokens, a 1x4 one with 1; both whole, then the first as text only
    img, txt, grid = [6, 4], [2, 1], [[1, 2, 3], [1, 1, 4]]
    cu, src = [0, 13, 20], [0] * 8 + [1] * 5 + [0] * 2 + [1] * 5
    t, h, w = orope.positions(cu, src, img, txt, grid)
    assert list(t) == [0, 0, 0, 0, 0, 0, 3, 4, 5, 5, 5, 5, 9, 0, 1, 2, 2, 2, 2, 6]
    assert list(h) == [0, 0, 0, 1, 1, 1, 3, 4, 5, 5, 5, 5, 9, 0, 1, 2, 2, 2, 2, 6]
    assert list(w) == [0, 1, 2, 0, 1, 2, 3, 4, 5, 6, 7, 8, 9, 0, 1, 2, 3, 4, 5, 6]


def test_frames_move_the_first_axis():
    pos = orope.positions([0, 9], [0] * 9, [8], [1], [[2, 2, 2]])
    assert pos.tolist() == [[0, 0, 0, 0, 1, 1, 1, 1, 2], [0, 0, 1, 1, 0, 0, 1, 1, 2], [0, 1, 0, 1, 0, 1, 0, 1, 2]]


def test_text_only_positions_are_the_builders():
    cu, img, txt = [0, 4], np.zeros(4, np.int32), np.array([3, 0, 5, 2], np.int32)
    lay = oseg.build(np.array(cu, np.int32), img, txt, 2, 1)
    pos = orope.positions(lay["cu_seqlens"], lay["tok_src_step"], img, txt, np.zeros((4, 3), int))
    assert all(np.array_equal(p, lay["tok_pos"]) for p in pos)


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_keeps_lengths_and_turns_back(interleaved):
    rng = np.random.default_rng(0)
    x, pos = rng.normal(size=(7, 3, 24)), rng.integers(-50, 5000, size=(3, 7))
    inv, axis = orope.frequencies(16, (2, 3, 3), 1e4)
    y = orope.rotate(x, pos, inv, axis, interleaved)
    assert np.array_equal(y[..., 16:], x[..., 16:])
    assert np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1))
    assert np.allclose(orope.rotate(y, pos, inv, axis, interleaved, back=True), x)


def test_scores_depend_on_differences_only():
    rng = np.random.default_rng(1)
    q, k = rng.normal(size=(2, 1, 1, 16))
    inv, axis = orope.frequencies(16, (2, 3, 3), 100.0)
    a, b = np.array([[5], [9], [2]]), np.array([[3], [4], [8]])
    dot = [(orope.rotate(q, a + s, inv, axis) * orope.rotate(k, b + s, inv, axis)).sum() for s in (0, 17)]
    assert np.isclose(dot[0], dot[1])


def test_gradient_against_differences():
    rng = np.random.default_rng(2)
    gather, t = np.array([0, 2, 1, 2, 2, 4]), 5
    pos, w = rng.integers(0, 40, size=(2, 6)), rng.normal(size=(6, 2, 16))
    inv, axis = orope.frequencies(16, (5, 3), 50.0)
    x = rng.normal(size=(t, 2, 16))
    f = lambda z: (orope.rotate(z[gather], pos, inv, axis) * w).sum()  # noqa: E731
    grad = orope.scatter(orope.rotate(w, pos, inv, axis, back=True), gather, t)
    for i in np.ndindex(t, 2, 16):
        if sum(i) % 5:
            continue
        d = np.zeros_like(x)
        d[i] = 1e-5
        assert abs((f(x + d) - f(x - d)) / 2e-5 - grad[i]) < 1e-8
    assert not grad[3].any()


def test_inverse_lists():
    off, tok = orope.inverse([3, 0, 3, 1, 0, 3], 5)
    assert off.tolist() == [0, 2, 3, 3, 6, 6] and tok.tolist() == [1, 4, 3, 0, 2, 5]
