"""Pins for oracle/distill.py: hand-worked values, the library's divergence, differences.  CPU only."""
import math

import numpy as np
import pytest
import torch

from oracle import distill as odis


def test_hand_worked():
    # a uniform student over four tokens; the teacher's two entries 3 : 1
    z = np.zeros((1, 4))
    loss, kl, g = odis.distill(z, [[2, 0]], [[math.log(3.0), 0.0]], [2.0])
    want = 0.75 * math.log(3) + 0.25 * math.log(1)   # p ln(p / 0.25)
    assert kl[0] == pytest.approx(want, abs=1e-14) and loss == pytest.approx(2 * want, abs=1e-14)
    np.testing.assert_allclose(g, [[2 * (0.25 - 0.25), 0.5, 2 * (0.25 - 0.75), 0.5]], atol=1e-14)


def test_a_full_list_is_the_library_s_divergence():
    rng = np.random.default_rng(0)
    z, t = rng.normal(size=(5, 9)) * 3, rng.normal(size=(5, 9)) * 3
    for temp in (1.0, 2.5):
        order = np.array([rng.permutation(9) for _ in range(5)])
        loss, kl, _ = odis.distill(z, order, np.take_along_axis(t, order, 1), np.ones(5), temperature=temp)
        p, q = (torch.log_softmax(torch.from_numpy(x / temp), 1) for x in (t, z))
        want = torch.nn.functional.kl_div(q, p, reduction="none", log_target=True).sum(1).numpy()
        np.testing.assert_allclose(kl, want, atol=1e-12)
        assert loss == pytest.approx(want.sum())


def test_gradient_by_differences_and_sum():
    rng = np.random.default_rng(5)
    z, t, w = rng.normal(size=(4, 7)), rng.normal(size=(6, 3)), np.array([0.5, 0.0, -1.0, 2.0])
    ids = np.array([[1, 5, 1], [0, 2, 3], [6, -1, 4], [-1, -1, -1], [2, 2, 2], [0, 6, 5]])
    rows = [0, 1, 2, 4]
    _, kl, g = odis.distill(z, ids, t, w, rows, 1.7)
    assert kl[1] == 0 and not g[1].any()
    np.testing.assert_allclose(g.sum(1), 0, atol=1e-14)
    for r in range(4):
        for v in range(7):
            f = []
            for step in (1e-6, -1e-6):
                x = z.copy()
                x[r, v] += step
                f.append(odis.distill(x, ids, t, w, rows, 1.7)[0])
            assert (f[0] - f[1]) / 2e-6 == pytest.approx(g[r, v], abs=1e-8)


def test_lists_without_entries():
    z = np.zeros((2, 3))
    loss, kl, g = odis.distill(z, [[-1, -1], [0, 1]], [[1.0, 2.0], [-math.inf, -math.inf]], [1.0, 1.0])
    assert loss == 0 and not kl.any() and not g.any()
