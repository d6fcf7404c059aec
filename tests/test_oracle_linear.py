"""Pins for oracle/linear.py: hand-worked values, the recurrence against the sums, differences, invariants.  CPU only."""
import math

import numpy as np
import pytest

from oracle import linear as olin


def draw(seed, n, hq, hkv, d):
    rng = np.random.default_rng(seed)
    return [rng.normal(size=(n, h, d)) for h in (hq, hkv, hkv, hq)]


def test_hand_worked():
    # one dim, decay 1/2: S = 2*3, then 6/2 + 1*5 = 8, then 4 + (-1)*2 = 2
    q, k, v = (np.array(x, float).reshape(3, 1, 1) for x in ([1, 2, 3], [2, 1, -1], [3, 5, 2]))
    g = np.array([math.log(0.5)])
    o, st = olin.walk(q, k, v, g, [0, 3], scale=1.0)
    np.testing.assert_allclose(o[:, 0, 0], [6, 16, 6], atol=1e-12)
    np.testing.assert_allclose(st, [[[[2.0]]]], atol=1e-12)
    o, st = olin.walk(q, k, v, g, [0, 1, 1, 3], state=np.full((3, 1, 1, 1), 4.0), scale=0.5)
    np.testing.assert_allclose(o[:, 0, 0], [(2 + 6) / 2, (2 + 5) * 2 / 2, (3.5 - 2) * 3 / 2], atol=1e-12)
    np.testing.assert_allclose(st[:, 0, 0, 0], [8, 4, 1.5], atol=1e-12)


@pytest.mark.parametrize("hq,hkv", [(1, 1), (4, 2), (3, 3), (6, 1)])
def test_sums_are_the_recurrence(hq, hkv):
    q, k, v, _ = draw(hq, 23, hq, hkv, 5)
    g, cu = -np.abs(np.random.default_rng(3).normal(size=hkv)), [0, 7, 7, 8, 23]
    st = np.random.default_rng(4).normal(size=(4, hkv, 5, 5))
    for s in (None, st):
        o, out = olin.walk(q, k, v, g, cu, s)
        r = olin.attn(q, k, v, g, cu, s)
        np.testing.assert_allclose(r["o"], o, atol=1e-12)
        np.testing.assert_allclose(r["state"], out, atol=1e-12)
        assert (r["o_abs"] >= np.abs(o) - 1e-12).all() and (r["state_abs"] >= np.abs(out) - 1e-12).all()
    b, t, x = 8, 20, hq - 1
    want, size = olin.row(q, k, v, g[-1], b, t, x, hkv - 1)
    r = olin.attn(q, k, v, g, cu)
    np.testing.assert_allclose(want, r["o"][t, x], atol=1e-12)
    np.testing.assert_allclose(size, r["o_abs"][t, x], atol=1e-12)


def test_gradients_by_differences():
    q, k, v, do = draw(9, 12, 4, 2, 3)
    g, cu = np.array([-0.3, 0.0]), [0, 5, 12]
    r = olin.grads(q, k, v, do, g, cu)
    rng = np.random.default_rng(1)
    for name, x in (("dq", q), ("dk", k), ("dv", v)):
        for _ in range(12):
            at = tuple(int(rng.integers(0, n)) for n in x.shape)
            keep, f = x[at], []
            for step in (1e-5, -1e-5):
                x[at] = keep + step
                f.append((olin.walk(q, k, v, g, cu)[0] * do).sum())
            x[at] = keep
            assert (f[0] - f[1]) / 2e-5 == pytest.approx(r[name][at], rel=1e-6, abs=1e-8)


def test_two_calls_are_one():
    q, k, v, _ = draw(2, 30, 2, 1, 4)
    g = np.array([-0.1])
    o, st = olin.walk(q, k, v, g, [0, 30])
    a, mid = olin.walk(q[:11], k[:11], v[:11], g, [0, 11])
    b, end = olin.walk(q[11:], k[11:], v[11:], g, [0, 19], state=mid)
    np.testing.assert_allclose(np.concatenate([a, b]), o, atol=1e-12)
    np.testing.assert_allclose(end, st, atol=1e-12)
