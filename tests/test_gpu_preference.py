"""GPU tests of the preference loss on pairs of sentences against the 64-bit oracle.

Tolerances: a margin is a 64-bit difference rounded once, 2^-24 of it; x carries another 2^-24, exponentials and logarithms 2^-22:
loss 2^-21 (1 + |x|); a gradient is a 64-bit sum of 32-bit weights, each good to 2^-21 (1 + |x|) beta |g|, rounded once.
"""
import numpy as np
import pytest

from oracle import losses_oracle as LO
from operator_util import close, guarded, put, rounded, values
from paper_2310_14997_amd import binding as bd

pytestmark = pytest.mark.gpu


def inputs(B, n, seed=0):
    rng = np.random.default_rng(seed + 17 * B + n)
    z = rounded(-150 + 40 * rng.normal(size=B), False)
    ref = rounded(z + 5 * rng.normal(size=B), False)
    c, r = rng.integers(0, B, size=n).astype(np.int32), rng.integers(0, B, size=n).astype(np.int32)
    c[rng.random(n) < 0.1] = -1
    r[rng.random(n) < 0.1] = -2
    return z, ref, c, r, rounded(rng.normal(size=n), False)


@pytest.mark.parametrize("B,n", [(1, 1), (2, 1), (3, 0), (5, 63), (64, 32), (63, 65), (17, 1000), (960, 8192), (1025, 300), (65536, 70)])
def test_losses_and_gradients(B, n):
    import torch
    f = torch.float32
    for ref_there, weights, beta, eps in ((True, True, 0.1, 0.1), (False, False, 2.0, 0.0), (True, False, 0.5, 1.0)):
        print("case preference", B, n, ref_there, eps, flush=True)
        z, ref, c, r, g = inputs(B, n)
        ref, g = ref if ref_there else None, g if weights else None
        loss, margin, grad = LO.preference(z, ref, c, r, beta, eps, g)
        x = beta * margin
        b32 = float(np.float32(beta))
        tl = 2.0 ** -21 * (1 + np.abs(x)) + 2.0 ** -23 * np.abs(loss)
        w = 2.0 ** -21 * (1 + np.abs(x)) * b32 * (1.0 if g is None else np.abs(g))
        tg = 2.0 ** -22 * np.abs(grad)
        np.add.at(tg, np.maximum(c, 0), w)
        np.add.at(tg, np.maximum(r, 0), w)
        tz, tr, tc, tj = put(z, f), None if ref is None else put(ref, f), put(c, torch.int32), put(r, torch.int32)
        tw = None if g is None else put(g, f)
        o = [guarded((n,), f, 1), guarded((n,), f, 2), guarded((B,), f, 3)]
        l, m, gz = (t for t, _ in o)
        gz.fill_(float("nan"))
        bd.spcfg_preference_forward_backward(tz, tr, tc, tj, beta, eps, tw, l, m, gz)
        close("loss", values(l), loss, tl)
        close("margin", values(m), margin, 2.0 ** -24 * np.abs(margin))
        close("gradient", values(gz), grad, tg)
        kept = [t.clone() for t in (l, m, gz)]
        for t in (l, m, gz):
            t.fill_(float("nan"))
        bd.spcfg_preference_forward(tz, tr, tc, tj, beta, eps, l, m)
        bd.spcfg_preference_backward(tz, tr, tc, tj, beta, eps, tw, gz)
        assert all(torch.equal(a, b) for a, b in zip(kept, (l, m, gz)))
        for _, ok in o:
            ok()


def test_sentences_that_cannot_be_derived_and_bad_indices():
    import torch
    inf, nan = float("inf"), float("nan")
    f = torch.float32
    z = put(np.array([-10.0, -inf, -inf, -12.0, nan, -9.0]), f)
    c = put(np.array([0, 1, 1, 0, 3, 5, 4], np.int32), torch.int32)
    r = put(np.array([3, 0, 2, 1, 6, 5, 1], np.int32), torch.int32)
    l, m, g = torch.empty(7, device="cuda:0"), torch.empty(7, device="cuda:0"), torch.empty(6, device="cuda:0")
    bd.spcfg_preference_forward_backward(z, None, c, r, 1.0, 0.0, None, l, m, g)
    loss, margin, grad = values(l), values(m), values(g)
    assert abs(loss[0] - np.log1p(np.exp(-2.0))) < 1e-6
    assert loss[1] == inf and margin[1] == -inf     # the better sentence cannot be derived
    assert loss[2] == 0 and margin[2] == 0          # neither can: left out
    assert loss[3] == 0 and margin[3] == inf
    assert np.isnan(loss[4]) and np.isnan(margin[4])  # an index past the last sentence
    assert abs(loss[5] - np.log(2.0)) < 1e-6 and margin[5] == 0 and grad[5] == 0
    assert np.isnan(loss[6])                        # a log Z that is no number
    s = 1 / (1 + np.exp(2.0))
    assert abs(grad[0] - (1 - s)) < 1e-6            # -s from the first pair, +1 from the second
    assert np.isnan(grad[3]) and np.isnan(grad[4]) and np.isnan(grad[1]) and grad[2] == 0


def test_graphs():
    import torch
    f = torch.float32
    z, ref, c, r, w = inputs(200, 500)
    tz, tr, tc, tj, tw = put(z, f), put(ref, f), put(c, torch.int32), put(r, torch.int32), put(w, f)
    l, m, g = torch.empty(500, device="cuda:0"), torch.empty(500, device="cuda:0"), torch.empty(200, device="cuda:0")
    step = lambda: bd.spcfg_preference_forward_backward(tz, tr, tc, tj, 0.1, 0.1, tw, l, m, g)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        tz.add_(tr, alpha=-0.25)
        for t in (l, m, g):
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (l, m, g)]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (l, m, g)))
