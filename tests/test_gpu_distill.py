"""GPU tests of distillation from a teacher's top entries against the 64-bit oracle.

Tolerances from the roundings on the way, with u = 2^-24: the sum of exponentials is good to 2^-19 (its argument 3 u |x| e^x
per term, its power 2 u, at most 100 additions on the way to the result), so lse is good to 2^-19 + u |lse|; p to 2^-20; the loss's
terms are summed in 64 bits: tau^2 (2^-19 + 2^-20 sum p (|log p| + |log q|)) + u |loss|; a gradient to
|g| tau (2^-18 q + 2^-20 p) plus half a step of its type (2^-24, bf16 2^-8).  From a kept lse, rounded to 32 bits, q is off by
another 2^-23 (|lse| + |s| / tau).  Numbers below the smallest normal one of 32 bits, 2^-126, may come out as 0: a softmax's entry
before it is scaled, and the result.
"""
import numpy as np
import pytest

from oracle import losses_oracle as LO
from operator_util import close, guarded, put, rounded, values
from paper_2310_14997_amd import binding as bd

pytestmark = pytest.mark.gpu


def dtype(bf16):
    import torch
    return torch.bfloat16 if bf16 else torch.float32


def scratch(R, V):
    import torch
    n = bd.spcfg_distill_workspace_bytes(R, V)
    return torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda:0") if n else None


def inputs(R, V, k, bf16, seed=0, absent=0.3, twice=False):
    rng = np.random.default_rng(seed * 100003 + R * 31 + V + k)
    s = rounded(2 * rng.normal(size=(R, V)), bf16)
    t = rounded(-np.sort(-3 * rng.normal(size=(R, k)), axis=1), bf16)
    if twice:
        ids = rng.integers(0, max(1, V // 2), size=(R, k))
    else:
        ids = np.stack([rng.choice(V, size=k, replace=False) for _ in range(R)])
    ids = np.where(rng.random((R, k)) < absent, -1, ids).astype(np.int32)
    ids[R // 2] = -1  # a row without entries
    g = rng.random(R) + 0.1
    if R > 2:
        g[R - 1] = 0.0
    return s, t, ids, rounded(g, False)


def check(d, tau, bf16, shift=0):
    import torch
    s, t, ids, g = d
    (R, V), k = s.shape, ids.shape[1]
    loss, lse, grad = LO.distill(s, t, ids, tau, g)
    q = np.exp(s / tau - lse[:, None])
    p_log = np.zeros(R)
    p_at = np.zeros((R, V))
    for r in range(R):
        at = ids[r][ids[r] >= 0]
        if not len(at):
            continue
        a = t[r][ids[r] >= 0] / tau
        lp = a - a.max() - np.log(np.exp(a - a.max()).sum())
        np.add.at(p_at[r], at, np.exp(lp))
        p_log[r] = (np.exp(lp) * (np.abs(lp) + np.abs(s[r][at] / tau) + abs(lse[r]))).sum()
    tl = tau ** 2 * (2.0 ** -19 + 2.0 ** -20 * p_log) + 2.0 ** -24 * np.abs(loss)
    te = 2.0 ** -19 + 2.0 ** -23 * np.abs(lse)
    tg = np.abs(g)[:, None] * tau * (2.0 ** -18 * q + 2.0 ** -20 * p_at) + (2.0 ** -8 if bf16 else 2.0 ** -24) * np.abs(grad)
    tg = tg + 2.0 ** -126 * (1 + np.abs(g)[:, None] * tau)
    kept = np.abs(g)[:, None] * tau * q * 2.0 ** -23 * (np.abs(lse)[:, None] + np.abs(s) / tau)
    f = torch.float32
    ts, tt, ti, tw = put(s, dtype(bf16), shift), put(t, dtype(bf16), shift), put(ids, torch.int32, shift), put(g, f, shift)
    ws = scratch(R, V)
    o1, ok1 = guarded((R,), f, shift)
    o2, ok2 = guarded((R,), f, shift)
    gr, ok3 = guarded((R, V), dtype(bf16), shift)
    bd.spcfg_distill_forward(ts, tt, ti, tau, o1, o2, ws)
    close("loss", values(o1), loss, tl)
    close("lse", values(o2), lse, te)
    bd.spcfg_distill_backward(ts, tt, ti, tau, o2, tw, gr)
    close("gradient from lse", values(gr), grad, tg + kept)
    first = o1.clone()
    for x in (o1, o2, gr):
        x.fill_(float("nan"))
    bd.spcfg_distill_forward_backward(ts, tt, ti, tau, tw, o1, o2, gr, ws)
    close("loss (both)", values(o1), loss, tl)
    close("lse (both)", values(o2), lse, te)
    close("gradient (both)", values(gr), grad, tg)
    assert torch.equal(first, o1)
    empty = (ids < 0).all(axis=1) | (g == 0)
    assert np.all(values(gr)[empty] == 0) and np.all(values(o1)[(ids < 0).all(axis=1)] == 0)
    for ok in (ok1, ok2, ok3):
        ok()


SIZES = [(1, 1, 1), (2, 2, 2), (5, 3, 2), (60, 200, 8), (7, 1021, 64), (4, 1025, 3), (33, 4093, 17), (3, 4099, 100), (19, 10000, 64),
         (2, 16381, 256), (3, 16390, 5), (2, 32767, 31), (1, 131071, 1024), (5, 70001, 128), (600, 300, 300)]


@pytest.mark.parametrize("bf16", [False, True], ids=["fp32", "bf16"])
@pytest.mark.parametrize("R,V,k", SIZES)
def test_losses_and_gradients(R, V, k, bf16):
    print("case distill", R, V, k, bf16, flush=True)
    check(inputs(R, V, k, bf16), 1.0 if k % 2 else 2.5, bf16)


@pytest.mark.parametrize("bf16", [False, True], ids=["fp32", "bf16"])
@pytest.mark.parametrize("R,V,k", [(5, 333, 40), (6, 4101, 40), (3, 40001, 40)])
def test_alignments_and_equal_ids(R, V, k, bf16):
    for shift in (1, 2, 5):
        print("case distill shift", R, V, k, bf16, shift, flush=True)
        check(inputs(R, V, k, bf16, seed=shift), 1.0, bf16, shift)
    check(inputs(R, V, k, bf16, seed=9, twice=True), 4.0, bf16)


def test_peaked_and_far_scores():
    """One score far above the others, scores that differ by thousands: exponentials that vanish."""
    for V in (50, 5000, 40000):
        s, t, ids, g = inputs(4, V, 6, False, seed=3)
        s[0] *= 500.0
        s[1, 7] = 300.0
        t[2] *= 300.0
        check((rounded(s, False), rounded(t, False), ids, g), 1.0, False)


@pytest.mark.parametrize("V", [40, 6000, 50000])
@pytest.mark.parametrize("bf16", [False, True], ids=["fp32", "bf16"])
def test_values_that_are_not_finite(V, bf16):
    import torch
    inf, nan = float("inf"), float("nan")
    R, k = 9, 3
    s = np.zeros((R, V))
    t = np.zeros((R, k))
    ids = np.tile(np.array([[1, 2, 3]], np.int32), (R, 1))
    s[0, 2] = -inf          # a student that rules out what the teacher keeps
    s[1, 5] = -inf          # ... or something else
    t[2, 1] = -inf          # an absent entry
    t[3] = -inf             # nothing there
    ids[4, 0] = V           # out of range
    s[5, 4] = nan
    t[6, 2] = nan
    s[7] = -inf
    ids[8] = -1             # nothing there; its scores are not looked at for the gradient
    s[8, 3] = nan
    f = torch.float32
    ts, tt, ti = put(s, dtype(bf16)), put(t, dtype(bf16)), put(ids, torch.int32)
    ws, l, e, g = scratch(R, V), torch.empty(R, device="cuda:0"), torch.empty(R, device="cuda:0"), torch.empty(R, V, dtype=dtype(bf16), device="cuda:0")
    for which in ("both", "backward"):
        if which == "both":
            bd.spcfg_distill_forward_backward(ts, tt, ti, 1.0, None, l, e, g, ws)
        else:
            g.fill_(7.0)
            bd.spcfg_distill_backward(ts, tt, ti, 1.0, e, None, g)
        loss, grad = values(l), values(g)
        step = 2.0 ** -7 if bf16 else 1e-5
        assert loss[0] == inf and np.all(np.isfinite(grad[0])) and abs(grad[0, 2] + 1 / 3) < step and grad[0, 9] > 0
        want = np.log(1 / 3) + np.log(V - 1)
        assert abs(loss[1] - want) < 1e-5 and grad[1, 5] == 0 and abs(grad[1, 1] - (1 / (V - 1) - 1 / 3)) < step
        want = np.log(1 / 2) + np.log(V)
        assert abs(loss[2] - want) < 1e-5 and abs(grad[2, 2] - 1 / V) < step / V and abs(grad[2, 1] - (1 / V - 0.5)) < step
        assert loss[3] == 0 and np.all(grad[3] == 0)
        for r in (4, 5, 6, 7):
            assert np.isnan(loss[r]) and np.all(np.isnan(grad[r])), r
        assert loss[8] == 0 and np.all(grad[8] == 0)
    # a weight of zero takes a row out, whatever is in it
    w = torch.zeros(R, device="cuda:0")
    bd.spcfg_distill_forward_backward(ts, tt, ti, 1.0, w, l, e, g, ws)
    assert np.all(values(g) == 0)


def test_no_rows_and_graphs():
    import torch
    f = torch.float32
    z = lambda *s: torch.empty(*s, device="cuda:0")
    i = torch.empty(0, 4, dtype=torch.int32, device="cuda:0")
    bd.spcfg_distill_forward_backward(z(0, 9), z(0, 4), i, 1.0, None, z(0), z(0), z(0, 9), None)
    for R, V in ((6, 900), (3, 60000)):
        s, t, ids, g = inputs(R, V, 12, False, seed=4)
        ts, tt, ti, tw = put(s, f), put(t, f), put(ids, torch.int32), put(g, f)
        l, e, gr, ws = z(R), z(R), z(R, V), scratch(R, V)
        step = lambda: bd.spcfg_distill_forward_backward(ts, tt, ti, 2.0, tw, l, e, gr, ws)
        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        for turn in range(3):
            ts.mul_(0.75)
            for x in (l, e, gr):
                x.fill_(float("nan"))
            graph.replay()
            torch.cuda.synchronize()
            got = [x.clone() for x in (l, e, gr)]
            step()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, (l, e, gr))), (R, V, turn)


def test_tables_of_more_than_32_bits_of_bytes():
    """Rows past 4 GB and 2^31 elements, in a table of 5.4 GB: the last rows against the oracle, the others by what they add up to."""
    import torch
    for R, V in ((20600, 131072), (131090, 20480)):
        print("case distill far offsets", R, V, flush=True)
        dev, b16, k = "cuda:0", torch.bfloat16, 7
        g = torch.Generator(device=dev)
        g.manual_seed(R)
        s = torch.empty(R, V, dtype=b16, device=dev)
        for r in range(0, R, 4096):
            s[r:r + 4096] = torch.randn(min(4096, R - r), V, generator=g, device=dev).to(b16)
        t = torch.randn(R, k, generator=g, device=dev).to(b16)
        ids = torch.randint(0, V, (R, k), generator=g, device=dev, dtype=torch.int32)
        l, e, gr = torch.empty(R, device=dev), torch.empty(R, device=dev), torch.empty_like(s)
        bd.spcfg_distill_forward_backward(s, t, ids, 1.0, None, l, e, gr, scratch(R, V))
        pick = torch.tensor([0, 1, R // 2, R - 2, R - 1], device=dev)
        loss, lse, grad = LO.distill(values(s[pick]), values(t[pick]), ids[pick].cpu().numpy(), 1.0)
        close("loss", values(l[pick]), loss, 2.0 ** -19 + 2.0 ** -17 * np.abs(loss))
        close("lse", values(e[pick]), lse, 2.0 ** -19 + 2.0 ** -23 * np.abs(lse))
        close("gradient", values(gr[pick]), grad, 2.0 ** -8 * np.abs(grad) + 2.0 ** -18 * np.exp(values(s[pick]) - lse[:, None]) + 2.0 ** -20 * (grad < 0))
        bd.spcfg_distill_backward(s, t, ids, 1.0, e, None, gr)
        close("gradient from lse", values(gr[pick]), grad, (2.0 ** -8 + 2.0 ** -16) * np.abs(grad) + 2.0 ** -16 * np.exp(values(s[pick]) - lse[:, None]) + 2.0 ** -20 * (grad < 0))
        del s, gr


@pytest.mark.parametrize("bf16", [False, True], ids=["fp32", "bf16"])
@pytest.mark.parametrize("R,V,k", [(20, 70001, 16), (50, 70001, 16), (70, 70001, 16), (520, 4203, 5), (520, 9001, 5), (700, 250, 9)])
def test_many_rows(R, V, k, bf16):
    """Parts of two, four and eight vectors a thread, rows whole in 256 threads, short rows of a wavefront each."""
    print("case distill rows", R, V, k, bf16, flush=True)
    check(inputs(R, V, k, bf16), 1.5, bf16)


@pytest.mark.parametrize("bf16", [False, True], ids=["fp32", "bf16"])
@pytest.mark.parametrize("V", [300, 5000, 40003])
def test_entries_side_by_side(V, bf16):
    """Every element of a stretch with an entry, some with two or more, and a row whose entries all have one id: twice the same."""
    import torch
    R, k = 5, 256
    s, t, ids, g = inputs(R, V, k, bf16, seed=4)
    order = np.random.default_rng(6).permutation(k)
    ids[0] = order
    ids[1] = V - 1 - order // 2
    ids[2] = 17
    ids[3] = np.where(order < 250, order % 5, -1)
    ids[4] = V - 1
    g[:] = 1.25
    # p of equal ids is added up in 64 bits and rounded once more: 2^-24 within the 2^-20 that an entry is allowed
    check((s, t, ids, g), 2.0, bf16, 1)
    ts, tt, ti = put(s, dtype(bf16)), put(t, dtype(bf16)), put(ids, torch.int32)
    l, e, ws = torch.empty(R, device="cuda:0"), torch.empty(R, device="cuda:0"), scratch(R, V)
    a, b = (torch.empty(R, V, dtype=dtype(bf16), device="cuda:0") for _ in range(2))
    for out in (a, b):
        bd.spcfg_distill_forward_backward(ts, tt, ti, 2.0, None, l, e, out, ws)
    assert torch.equal(a, b)
    for out in (a, b):
        bd.spcfg_distill_backward(ts, tt, ti, 2.0, e, None, out)
    assert torch.equal(a, b)
