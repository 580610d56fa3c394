"""GPU tests of distillation where it is easily wrong: low temperatures, whose lse is large.

Tolerances with u = 2^-24 as in test_gpu_distill.py, but for the gradient alone: the joint call's, bit for bit, where a workgroup holds a
row; of longer rows, the joint call's and u |lse| of q, the rounding of the kept lse (exponents are formed in 64 bits)."""
import numpy as np
import pytest

from oracle import losses_oracle as LO
from operator_util import close, put, values
from paper_2310_14997_amd import binding as bd
from test_gpu_distill import dtype, inputs, scratch

pytestmark = pytest.mark.gpu


def calls(s, t, ids, tau, g, bf16):
    """gradient of the joint call, gradient alone, lse"""
    import torch
    (R, V), f = s.shape, torch.float32
    ts, tt, ti = put(s, dtype(bf16)), put(t, dtype(bf16)), put(ids, torch.int32)
    tw = None if g is None else put(g, f)
    e = lambda *n, d=f: torch.full(n, float("nan"), dtype=d, device="cuda:0")
    loss, lse, both, alone = e(R), e(R), e(R, V, d=dtype(bf16)), e(R, V, d=dtype(bf16))
    bd.spcfg_distill_forward_backward(ts, tt, ti, tau, tw, loss, lse, both, scratch(R, V))
    bd.spcfg_distill_backward(ts, tt, ti, tau, lse, tw, alone)
    return both, alone, lse


@pytest.mark.parametrize("bf16", [False, True], ids=["fp32", "bf16"])
@pytest.mark.parametrize("V", [300, 900, 5000, 16000, 40000])
@pytest.mark.parametrize("tau,by", [(0.01, 1.0), (0.01, 14.0), (1.0, 300.0)])
def test_gradients_alone_at_low_temperatures(V, bf16, tau, by):
    """|lse| up to some thousands; in fp32 the rows' q add up to 1 within the tolerance too, which an error of one sign would break."""
    import torch
    R, k = 6, 8
    print("case distill low temperature", V, bf16, tau, by, flush=True)
    s, t, ids, g = inputs(R, V, k, bf16, seed=8)
    s, t = (np.clip(by * x, -5 * by, 5 * by) for x in (s, t))
    if bf16:
        s, t = (torch.from_numpy(x).to(torch.bfloat16).double().numpy() for x in (s, t))
    s[0], s[1] = np.float32(4.7 * by) if not bf16 else 4.0 * by, s[1] / 64  # a row of equal scores, a row of scores close together
    s, t = (torch.from_numpy(x).to(dtype(bf16)).double().numpy() for x in (s, t))  # the values that the call sees
    both, alone, lse = calls(s, t, ids, tau, g, bf16)
    if V <= 16000:
        assert torch.equal(both, alone)
    _, want_lse, grad = LO.distill(s, t, ids, tau, g)
    q = np.exp(s / tau - want_lse[:, None])
    p = q - grad / np.where(g == 0, 1.0, g)[:, None] / tau
    tg = np.abs(g)[:, None] * tau * (2.0 ** -18 * q + 2.0 ** -20 * np.abs(p)) + (2.0 ** -8 if bf16 else 2.0 ** -24) * np.abs(grad) \
        + 2.0 ** -126 * (1 + np.abs(g)[:, None] * tau)
    # exponents, (s - max) / tau of q and (t - max) / tau = log p + log sum of p, the sum at most k, are rounded at 2^-24 of themselves
    # three times: at a low temperature that is more than the 2^-18 and 2^-20 above
    x_p = np.where(np.abs(p) > 1e-300, np.log(k) - np.log(np.maximum(np.abs(p), 1e-300)), 0.0)
    tg = tg + np.abs(g)[:, None] * tau * 3 * 2.0 ** -24 * (q * (s.max(1, keepdims=True) - s) / tau + np.abs(p) * x_p)
    close("both", values(both), grad, tg)
    kept = 2.0 ** -24 * np.abs(want_lse)[:, None] * (V > 16000)
    close("alone", values(alone), grad, tg + np.abs(g)[:, None] * tau * q * kept)
    if not bf16:
        rows = (ids >= 0).any(axis=1) & (g != 0)
        off = np.abs(values(alone)[rows].sum(1)) / (tau * g[rows])
        assert np.all(off <= 2.0 ** -17 + kept[rows, 0]), (off, kept[rows, 0])


@pytest.mark.parametrize("V", [40, 6000, 50000])
def test_temperatures_whose_lse_does_not_fit(V):
    """lse is 5 / 1e-38: the gradient is that of the joint call where a workgroup holds the row, and NaN, not zeros, where it does not."""
    import torch
    rng = np.random.default_rng(3)
    s = rng.integers(-5, 5, size=(3, V)).astype(np.float64)
    s[:, 7] = 5.0
    t, ids = np.zeros((3, 2)), np.array([[7, 9], [11, -1], [-1, -1]], np.int32)
    g = np.full(3, 2.0 ** 120)
    both, alone, lse = calls(s, t, ids, 1e-38, g, False)
    assert bool(torch.isinf(lse).all())
    by = 2.0 ** 120 * np.float32(1e-38)
    want = np.zeros((3, V))
    want[0, 7], want[0, 9], want[1, 7], want[1, 11] = 0.5 * by, -0.5 * by, by, -by
    close("both", values(both), want, 2.0 ** -22 * np.abs(want))
    if V <= 16000:
        assert torch.equal(both, alone)
    else:
        assert bool(torch.isnan(alone[:2]).all()) and not bool(alone[2].any())


@pytest.mark.parametrize("V", [40, 6000, 50000])
@pytest.mark.parametrize("bf16", [False, True], ids=["fp32", "bf16"])
def test_padding_by_scores_of_minus_infinity(V, bf16):
    """Entries that pad a row, with a score of -inf and any id, one past the last among them, are absent: as with an id of -1."""
    import torch
    R, k, f = 4, 6, torch.float32
    s, t, ids, g = inputs(R, V, k, bf16, seed=2, absent=0.0)
    ids[0, 2:], ids[1, 5], ids[2] = -1, -1, -1
    ids[3] = [1, 0, 9, 5, 7, 3]
    padded, scores = ids.copy(), t.copy()
    padded[0, 2:], padded[1, 5], padded[2] = V, 2 ** 31 - 1, [V, V + 1, 0, 3, V, -5]
    scores[ids < 0] = -np.inf
    one, _, lse_one = calls(s, t, ids, 2.0, g, bf16)
    two, alone, lse_two = calls(s, scores, padded, 2.0, g, bf16)
    assert bool(torch.isfinite(one).all()) and torch.equal(one, two) and torch.equal(lse_one, lse_two)
    assert bool(torch.isfinite(alone).all()) and not bool(two[2].any())
    out = [torch.empty(R, device="cuda:0") for _ in range(4)]
    ts = put(s, dtype(bf16))
    bd.spcfg_distill_forward(ts, put(t, dtype(bf16)), put(ids, torch.int32), 2.0, out[0], out[1], scratch(R, V))
    bd.spcfg_distill_forward(ts, put(scores, dtype(bf16)), put(padded, torch.int32), 2.0, out[2], out[3], scratch(R, V))
    assert torch.equal(out[0], out[2]) and torch.equal(out[1], out[3]) and float(out[0][2]) == 0.0


@pytest.mark.parametrize("V", [40, 1000, 6000, 50000])
@pytest.mark.parametrize("bf16", [False, True], ids=["fp32", "bf16"])
def test_rows_of_nothing_but_minus_infinity(V, bf16):
    """lse is the log of an empty sum; loss and gradient are NaN with entries and 0 without; a NaN in the row, or one finite score, counts."""
    import torch
    inf = np.inf
    s = np.full((5, V), -inf)
    s[2, V - 3], s[3, V // 2] = np.nan, -3.0
    s[4] = 0.0
    t, ids = np.zeros((5, 2)), np.tile(np.array([[1, 2]], np.int32), (5, 1))
    ids[1] = -1
    both, alone, lse = calls(s, t, ids, 2.0, None, bf16)
    loss, lse_alone = torch.empty(5, device="cuda:0"), torch.empty(5, device="cuda:0")
    bd.spcfg_distill_forward(put(s, dtype(bf16)), put(t, dtype(bf16)), put(ids, torch.int32), 2.0, loss, lse_alone, scratch(5, V))
    want_loss, want_lse, want = LO.distill(s[[0, 1, 3]], t[[0, 1, 3]], ids[[0, 1, 3]], 2.0)
    assert want_lse[0] == -inf and want_lse[1] == -inf and np.isnan(want_loss[0]) and want_loss[1] == 0 and want_loss[2] == inf
    for got in (values(lse), values(lse_alone)):
        assert got[0] == -inf and got[1] == -inf and np.isnan(got[2]) and got[3] == -1.5 and abs(got[4] - np.log(V)) < 2.0 ** -18
    got = values(loss)
    assert np.isnan(got[0]) and got[1] == 0 and np.isnan(got[2]) and got[3] == inf
    for g in (values(both), values(alone)):
        assert np.isnan(g[0]).all() and np.isnan(want[0]).all() and not g[1].any() and np.isnan(g[2]).all()
        step = 2.0 ** -8 if bf16 else 2.0 ** -24
        assert np.all(np.abs(g[3] - want[2]) <= step * np.abs(want[2]) + 2.0 ** -19 * 2)
