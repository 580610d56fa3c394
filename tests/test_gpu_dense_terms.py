"""GPU tests of what the header states of single terms and of activations' tails.

  fp32 products  sums of one term: off by at most 2^-21 of it in large forward products (two fp16 pieces of each value, either to 2^-23,
                 and lo lo of 2^-22 left out), 2^-23 in small ones (three bf16 pieces); and by 2^-23 of the sum so far for each matrix
                 instruction: of the result for the last one, 2^-8 of that for those before, which add the smaller pieces.
  gelu, z < 0    |z| e^x q t / 2, x = -z^2 / 2: x is off by 5.5 2^-24 of itself (0.7071 |z| 1.5, squared 3 and 1, log2 e times it 1.5),
                 the rest by 16 2^-24: q 6, power, reciprocal and its argument 2 each, four products.
  silu, z < 0    e^-z off by 1.5 2^-24 |z|, sum, reciprocal, product and power by 8 2^-24.
  z > 0          gelu is z - z h with h = erfc / 2 <= 1/2, whose error counts h / (1 - h) <= 1 times: 2.75 z^2 h / (1 - h) < 1, so 18 2^-24
                 with the difference's own; silu's counts e^-z / (1 + e^-z) <= 1/2 times: less.
Below 2^-126 |z| either may be 0.
"""
import math

import numpy as np
import pytest

from operator_util import close, put, values
from paper_2310_14997_amd import binding as bd
from test_gpu_dense import workspace

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("R,I,O,bound", [(2048, 512, 520, 2.0 ** -21), (40, 64, 48, 2.0 ** -23)])
def test_single_terms(R, I, O, bound):
    import torch
    rng = np.random.default_rng(1)
    full = lambda *s: (rng.uniform(1, 2, size=s) * 2.0 ** rng.integers(-6, 6, size=s) * rng.choice([-1, 1], size=s)).astype(np.float32)
    x, W, at = np.zeros((R, I), np.float32), full(O, I), rng.integers(0, I, size=R)
    x[np.arange(R), at] = full(R)
    cfg, y = bd.make_dense_config(R, I, O), torch.empty(R, O, device="cuda:0")
    bd.spcfg_dense_forward(cfg, put(x, torch.float32), put(W, torch.float32), None, None, y, None, workspace(cfg))
    want = x[np.arange(R), at].astype(np.float64)[:, None] * W.astype(np.float64)[:, at].T
    close("y", values(y), want, (bound + 1.1 * 2.0 ** -23) * np.abs(want))


def test_tails_of_activations():
    import torch
    z = np.concatenate([-np.geomspace(1e-6, 120.0, 40000), np.geomspace(1e-6, 120.0, 4000)]).astype(np.float32)
    ones = torch.ones(1, 1, device="cuda:0")
    for act in (bd.ACT_GELU, bd.ACT_SILU):
        cfg, y = bd.make_dense_config(len(z), 1, 1, activation=act), torch.empty(len(z), 1, device="cuda:0")
        pre = torch.empty(len(z), 1, device="cuda:0")
        bd.spcfg_dense_forward(cfg, put(z[:, None], torch.float32), ones, None, None, y, pre, workspace(cfg))
        z64 = values(pre)[:, 0]
        close("preact", z64, z.astype(np.float64), 2.0 ** -23 * np.abs(z))
        if act == bd.ACT_GELU:
            want, off = np.array([0.5 * v * math.erfc(-v / math.sqrt(2.0)) for v in z64]), 2.75 * z64 ** 2 + 16
        else:
            e = np.exp(-np.abs(z64))
            want, off = np.where(z64 < 0, z64 * e / (1 + e), z64 / (1 + e)), 1.5 * np.abs(z64) + 8
        close("y", values(y)[:, 0], want, 2.0 ** -24 * np.where(z64 < 0, off, 18) * np.abs(want) + 2.0 ** -126 * np.abs(z64))
