"""Pins of the losses' oracle: differences, values worked out by hand, rows and pairs that are left out."""
import numpy as np
import pytest

from oracle import losses_oracle as LO


@pytest.mark.parametrize("tau", [1.0, 2.5])
def test_distillation_gradients_are_differences(tau):
    rng = np.random.default_rng(5)
    s, t = rng.normal(size=(3, 6)), rng.normal(size=(3, 4))
    ids = np.array([[0, 3, 5, 1], [2, -1, 4, 2], [-1, -1, -1, -1]])  # one id twice, one row without entries
    w = np.array([0.5, 2.0, 3.0])
    _, _, g = LO.distill(s, t, ids, tau, w)
    h = 1e-6
    for i in np.ndindex(s.shape):
        keep = s[i]
        s[i] = keep + h
        up = (LO.distill(s, t, ids, tau)[0] * w).sum()
        s[i] = keep - h
        down = (LO.distill(s, t, ids, tau)[0] * w).sum()
        s[i] = keep
        assert abs((up - down) / (2 * h) - g[i]) < 1e-8
    assert np.all(g[2] == 0)


def test_distillation_of_a_row_from_itself_is_nothing():
    s = np.log(np.array([[1.0, 2.0, 5.0]]))
    loss, lse, g = LO.distill(s, s[:, [2, 0, 1]], np.array([[2, 0, 1]]), 1.0)
    assert abs(loss[0]) < 1e-15 and abs(lse[0] - np.log(8.0)) < 1e-15 and np.abs(g).max() < 1e-15
    loss, _, g = LO.distill(s, [[0.0]], np.array([[0]]), 1.0)  # all weight on a word of probability 1/8
    assert abs(loss[0] - np.log(8.0)) < 1e-15 and np.allclose(g, [[-7 / 8, 2 / 8, 5 / 8]], atol=1e-15)


def test_preference_gradients_are_differences():
    rng = np.random.default_rng(6)
    z, ref = rng.normal(size=5) * 3, rng.normal(size=5)
    c, r = np.array([0, 1, 1, 4, -1, 2]), np.array([1, 2, 3, 4, 2, -3])
    w = rng.random(6)
    for eps in (0.0, 0.2):
        loss, margin, g = LO.preference(z, ref, c, r, 0.7, eps, w)
        assert loss[4] == loss[5] == margin[4] == 0 and margin[3] == 0
        h = 1e-6
        for i in range(5):
            keep = z[i]
            z[i] = keep + h
            up = (LO.preference(z, ref, c, r, 0.7, eps)[0] * w).sum()
            z[i] = keep - h
            down = (LO.preference(z, ref, c, r, 0.7, eps)[0] * w).sum()
            z[i] = keep
            assert abs((up - down) / (2 * h) - g[i]) < 1e-8
    loss, _, _ = LO.preference([3.0, 1.0], None, [0], [1], 1.0, 0.0)
    assert abs(loss[0] - 0.1269280110429725) < 1e-15
