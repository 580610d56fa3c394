"""Pins of the dense-layer oracle: differences of the forward pass, and values worked out by hand."""
import numpy as np
import pytest

from oracle import network_oracle as NO


@pytest.mark.parametrize("kind", ["none", "relu", "gelu", "silu"])
def test_gradients_are_differences(kind):
    rng = np.random.default_rng(3)
    x, W, b, gy = rng.normal(size=(4, 5)), rng.normal(size=(3, 5)), rng.normal(size=3), rng.normal(size=(4, 3))
    _, z = NO.forward(x, W, b, kind=kind)
    assert np.abs(z).min() > 1e-3  # (no difference crosses relu's corner)
    gx, gW, gb = NO.backward(x, W, z, gy, kind)
    h = 1e-6
    for a, g in ((x, gx), (W, gW), (b, gb)):
        for i in np.ndindex(a.shape):
            keep = a[i]
            a[i] = keep + h
            up = (NO.forward(x, W, b, kind=kind)[0] * gy).sum()
            a[i] = keep - h
            down = (NO.forward(x, W, b, kind=kind)[0] * gy).sum()
            a[i] = keep
            assert abs((up - down) / (2 * h) - g[i]) < 1e-8


def test_residuals_and_known_values():
    y, z = NO.forward([[1.0, 2.0]], [[3.0, -4.0]], [0.5], [[10.0]], "relu")
    assert z[0, 0] == -4.5 and y[0, 0] == 10.0
    assert abs(NO.act(np.array(1.0), "gelu") - 0.8413447460685429) < 1e-15
    assert abs(NO.act(np.array(1.0), "silu") - 0.7310585786300049) < 1e-15
    gx, _, _ = NO.backward([[1.0]], [[2.0]], [[1.0]], [[3.0]], "relu", [[100.0]])
    assert gx[0, 0] == 106.0
