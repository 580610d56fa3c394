"""CPU oracle for the dense layers of the networks that make the rule scores.  TEST INFRASTRUCTURE ONLY.

    z = x W^T + bias,  y = act(z) + residual          act: "none", "relu", "gelu" (erf), "silu"

and the gradients of sum(grad_y * y) in x, W and bias, with z given, since that is what a forward pass keeps.  Double
precision, numpy; shares no code with the HIP path.  Pinned in tests/test_network_oracle.py (finite differences).
"""
from __future__ import annotations

import math

import numpy as np

_erf = np.vectorize(math.erf, otypes=[np.float64])


def _sigmoid(z):
    e = np.exp(-np.abs(z))
    return np.where(z >= 0, 1.0 / (1.0 + e), e / (1.0 + e))


def act(z, kind):
    if kind == "relu":
        return np.maximum(z, 0.0)
    if kind == "gelu":
        return 0.5 * z * (1.0 + _erf(z / math.sqrt(2.0)))
    if kind == "silu":
        return z * _sigmoid(z)
    return z


def act_slope(z, kind):
    if kind == "relu":
        return (z > 0).astype(np.float64)
    if kind == "gelu":
        return 0.5 * (1.0 + _erf(z / math.sqrt(2.0))) + z * np.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    if kind == "silu":
        s = _sigmoid(z)
        return s + z * s * (1.0 - s)
    return np.ones_like(z)


def forward(x, W, bias=None, residual=None, kind="none"):
    """(y, z)"""
    z = np.asarray(x, np.float64) @ np.asarray(W, np.float64).T
    if bias is not None:
        z = z + np.asarray(bias, np.float64)
    y = act(z, kind)
    return (y if residual is None else y + np.asarray(residual, np.float64)), z


def backward(x, W, z, grad_y, kind="none", grad_x_add=None):
    """(grad_x, grad_W, grad_bias)"""
    dz = np.asarray(grad_y, np.float64)
    if kind != "none":
        dz = dz * act_slope(np.asarray(z, np.float64), kind)
    gx = dz @ np.asarray(W, np.float64)
    if grad_x_add is not None:
        gx = gx + np.asarray(grad_x_add, np.float64)
    return gx, dz.T @ np.asarray(x, np.float64), dz.sum(0)
