"""GPU tests of the dense layers against the 64-bit oracle: both directions, types, activations, odd sizes and alignments,
what is left out, accumulation, other streams and captured graphs.

Tolerances, per element, from the roundings on the way:
  products   sums of K terms in steps of 16, at most six piece products each (fp32), every step off by at most 2^-23 of a
             partial sum; partial sums of terms with random signs stay below twice the root q of the terms' squares:
             2^-23 (16 + 6 K / 16) 2 q.  The pieces that fp32 operands drop are below 2^-23 of each term, within the 16.
  dz         32-bit slopes are good to 2^-21 (1 + |z|) of grad_y; for bf16 operands dz is rounded to bf16, 2^-8 of each term,
             terms of random signs: 4 (2^-8) q.
  results    half a step: 2^-8 (bf16) or 2^-24 (fp32) of the value; activations and the epilogue's sums 2^-21 of their terms.
"""
import numpy as np
import pytest

from oracle import network_oracle as NO
from operator_util import close, guarded, put, rounded, values
from paper_2310_14997_amd import binding as bd

pytestmark = pytest.mark.gpu

ACTS = {"none": bd.ACT_NONE, "relu": bd.ACT_RELU, "gelu": bd.ACT_GELU, "silu": bd.ACT_SILU}
TYPES = [("fp32", "fp32"), ("bf16", "bf16"), ("bf16", "fp32")]
U = 2.0 ** -23


def t_of(name):
    return bd.TYPE_BF16 if name == "bf16" else bd.TYPE_F32


def d_of(name):
    import torch
    return torch.bfloat16 if name == "bf16" else torch.float32


def half_step(name):
    return 2.0 ** -8 if name == "bf16" else 2.0 ** -24


def product_tol(A, B):
    """of A B^T"""
    K = A.shape[1]
    return U * (16 + 6 * K / 16) * 2 * np.sqrt((A * A) @ (B * B).T)


def workspace(cfg):
    import torch
    n = bd.spcfg_dense_workspace_bytes(cfg)
    return torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda:0") if n else None


def inputs(R, I, O, types, seed=0):
    rng = np.random.default_rng(1000 * seed + R * 7 + I * 3 + O)
    bi, bo = (t == "bf16" for t in types)
    d = dict(x=rounded(rng.normal(size=(R, I)), bi), W=rounded(rng.normal(size=(O, I)) * np.sqrt(2 / (I + O)), bi),
             bias=rounded(0.2 * rng.normal(size=O), bi), residual=rounded(rng.normal(size=(R, O)), bo),
             grad_y=rounded(rng.normal(size=(R, O)), bo), add=rounded(rng.normal(size=(R, I)), bi))
    return d


def check_forward(R, I, O, types, act, bias=True, residual=True, keep=True, shift=0, stream=None):
    d = inputs(R, I, O, types)
    ti, to = d_of(types[0]), d_of(types[1])
    cfg = bd.make_dense_config(R, I, O, t_of(types[0]), t_of(types[1]), ACTS[act])
    y, y_ok = guarded((R, O), to, shift)
    z, z_ok = guarded((R, O), to, shift)
    bd.spcfg_dense_forward(cfg, put(d["x"], ti, shift), put(d["W"], ti, shift), put(d["bias"], ti, shift) if bias else None,
                           put(d["residual"], to, shift) if residual else None, y, z if keep else None, workspace(cfg))
    want, wz = NO.forward(d["x"], d["W"], d["bias"] if bias else None, d["residual"] if residual else None, act)
    ez = product_tol(d["x"], d["W"]) + 2.0 ** -21 * (np.abs(wz) + np.abs(d["bias"]))
    ey = 1.2 * ez + 2.0 ** -21 * (1 + np.abs(wz) + np.abs(want)) + half_step(types[1]) * np.abs(want)
    close("y", values(y), want, ey)
    if keep:
        close("preact", values(z), wz, ez + half_step(types[1]) * np.abs(wz))
    y_ok()
    z_ok()


def check_backward(R, I, O, types, act, add=True, want=("x", "W", "b"), accumulate=False, shift=0):
    d = inputs(R, I, O, types, seed=1)
    ti, to = d_of(types[0]), d_of(types[1])
    z = rounded(d["x"] @ d["W"].T + d["bias"], types[1] == "bf16")
    cfg = bd.make_dense_config(R, I, O, t_of(types[0]), t_of(types[1]), ACTS[act],
                               bd.FLAG_ACCUMULATE_GRADS if accumulate else 0)
    gx, x_ok = guarded((R, I), ti, shift)
    gW, W_ok = guarded((O, I), ti, shift)
    gb, b_ok = guarded((O,), ti, shift)
    gW.fill_(0.5)
    gb.fill_(-0.25)
    bd.spcfg_dense_backward(cfg, put(d["x"], ti, shift), put(d["W"], ti, shift),
                            put(z, to, shift) if act != "none" else None, put(d["grad_y"], to, shift),
                            put(d["add"], ti, shift) if add else None, gx if "x" in want else None,
                            gW if "W" in want else None, gb if "b" in want else None, workspace(cfg))
    wx, wW, wb = NO.backward(d["x"], d["W"], z, d["grad_y"], act, d["add"] if add else None)
    dz = d["grad_y"] * NO.act_slope(z, act)
    off = 2.0 ** -21 * np.abs(d["grad_y"]) * (1 + np.abs(z)) * (act != "none")  # of dz before its rounding
    if types[0] == "bf16":
        off = off + 2.0 ** -8 * np.abs(dz)
    spread = lambda A, B: 4 * np.sqrt((A * A) @ (B * B))
    hs = half_step(types[0])
    if "x" in want:
        close("grad_x", values(gx), wx, product_tol(dz, d["W"].T) + spread(off, d["W"]) + (hs + 2.0 ** -22) * np.abs(wx) +
              2.0 ** -22 * np.abs(d["add"]))
    if "W" in want:
        wW = wW + (0.5 if accumulate else 0.0)
        close("grad_W", values(gW), wW, product_tol(dz.T, d["x"].T) + spread(off.T, d["x"]) + (hs + 2.0 ** -22) * (np.abs(wW) + 1))
    if "b" in want:
        one = np.ones((R, 1))
        wb = wb + (-0.25 if accumulate else 0.0)
        close("grad_bias", values(gb), wb, (product_tol(dz.T, one.T) + spread(off.T, one))[:, 0] + (hs + 2.0 ** -22) * (np.abs(wb) + 1))
    for ok in (x_ok, W_ok, b_ok):
        ok()


SIZES = [(1, 1, 1), (1, 7, 3), (2, 16, 33), (3, 64, 32), (33, 100, 31), (64, 64, 64), (30, 512, 512), (129, 48, 1000),
         (257, 130, 65), (300, 520, 264), (1, 4096, 100), (1000, 1, 9), (9, 2000, 1)]


@pytest.mark.parametrize("types", TYPES, ids="-".join)
@pytest.mark.parametrize("R,I,O", SIZES)
def test_forward(R, I, O, types):
    print("case dense forward", R, I, O, types, flush=True)
    for act in ACTS:
        check_forward(R, I, O, types, act)


@pytest.mark.parametrize("types", TYPES, ids="-".join)
@pytest.mark.parametrize("R,I,O", SIZES)
def test_backward(R, I, O, types):
    print("case dense backward", R, I, O, types, flush=True)
    for act in ACTS:
        check_backward(R, I, O, types, act)


# sizes of more work: whole and ragged tiles along each side, long sums with few rows, few columns, few inputs
LARGE = [(2048, 512, 512), (1025, 264, 1111), (130, 2050, 700), (4100, 72, 130), (96, 1024, 6000), (2500, 640, 40),
         (777, 333, 1999), (2050, 520, 4104), (100, 4000, 1000), (8200, 512, 512)]


@pytest.mark.parametrize("types", TYPES, ids="-".join)
@pytest.mark.parametrize("R,I,O", LARGE)
def test_larger(R, I, O, types):
    print("case dense larger", R, I, O, types, flush=True)
    check_forward(R, I, O, types, "gelu")
    check_forward(R, I, O, types, "none", bias=False, residual=False, keep=False)
    check_backward(R, I, O, types, "silu")
    check_backward(R, I, O, types, "none", add=False)


@pytest.mark.parametrize("types", TYPES, ids="-".join)
def test_wide(types):
    """More tiles than CUs and long sums; the reference is 64-bit arithmetic on the GPU, over a sample of rows and columns."""
    import torch
    R, I, O = 4100, 2056, 4104
    print("case dense wide", types, flush=True)
    g = torch.Generator(device="cuda:0")
    g.manual_seed(7)
    n = lambda *s: torch.randn(*s, generator=g, device="cuda:0")
    ti, to = d_of(types[0]), d_of(types[1])
    x, W, b = n(R, I).to(ti), (n(O, I) * 0.02).to(ti), n(O).to(ti)
    r, gy = n(R, O).to(to), n(R, O).to(to)
    cfg = bd.make_dense_config(R, I, O, t_of(types[0]), t_of(types[1]), bd.ACT_RELU)
    ws = workspace(cfg)
    y, z = torch.empty(R, O, dtype=to, device="cuda:0"), torch.empty(R, O, dtype=to, device="cuda:0")
    bd.spcfg_dense_forward(cfg, x, W, b, r, y, z, ws)
    gx, gW, gb = (torch.full(s, float("nan"), dtype=ti, device="cuda:0") for s in ((R, I), (O, I), (O,)))
    bd.spcfg_dense_backward(cfg, x, W, z, gy, None, gx, gW, gb, ws)
    rows = torch.cat([torch.arange(0, R, 37), torch.arange(R - 5, R)]).cuda()
    cols = torch.cat([torch.arange(0, O, 41), torch.arange(O - 5, O)]).cuda()
    D = lambda t: t.double()
    want_z = D(x)[rows] @ D(W).t() + D(b)
    q = torch.sqrt((D(x)[rows] ** 2) @ (D(W) ** 2).t())
    ez = (U * (16 + 6 * I / 16) * 2 * q + 2.0 ** -21 * (want_z.abs() + D(b).abs())).cpu().numpy()
    close("preact", values(z[rows]), want_z.cpu().numpy(), ez + half_step(types[1]) * want_z.abs().cpu().numpy())
    want = want_z.clamp(min=0) + D(r)[rows]
    close("y", values(y[rows]), want.cpu().numpy(), ez + (2.0 ** -21 + half_step(types[1])) * want.abs().cpu().numpy())
    dz = D(gy) * (D(z) > 0)
    lossy = 4 * 2.0 ** -8 if types[0] == "bf16" else 0.0
    for name, got, A, B, K in (("grad_x", gx[rows], dz[rows], D(W), O), ("grad_W", gW[cols], dz[:, cols].t(), D(x), R)):
        want, q = A @ B, torch.sqrt((A ** 2) @ (B ** 2))
        tol = (U * (16 + 6 * K / 16) * 2 + lossy) * q + (half_step(types[0]) + 2.0 ** -22) * want.abs()
        close(name, values(got), want.cpu().numpy(), tol.cpu().numpy())
    want, q = dz.sum(0), torch.sqrt((dz ** 2).sum(0))
    close("grad_bias", values(gb), want.cpu().numpy(),
          (U * (16 + 6 * R / 16) * 2 * q + (half_step(types[0]) + 2.0 ** -22) * want.abs()).cpu().numpy())


@pytest.mark.parametrize("types", TYPES, ids="-".join)
@pytest.mark.parametrize("R,I,O", [(70, 64, 96), (1200, 520, 1040)])
def test_options_and_alignments(R, I, O, types):
    print("case dense options", R, I, O, types, flush=True)
    for bias, residual, keep in ((False, False, False), (True, False, False), (False, True, True), (False, False, True)):
        check_forward(R, I, O, types, "relu", bias, residual, keep)
    for want in (("x",), ("W",), ("W", "b"), ("x", "W")):
        check_backward(R, I, O, types, "relu", add="x" in want, want=want)
    check_backward(R, I, O, types, "gelu", accumulate=True)
    check_backward(R, I, O, types, "none", accumulate=True, add=False)
    for shift in (1, 3):
        check_forward(R, I, O, types, "silu", shift=shift)
        check_backward(R, I, O, types, "silu", shift=shift)


@pytest.mark.parametrize("types", TYPES, ids="-".join)
def test_no_rows(types):
    import torch
    check_forward(0, 5, 4, types, "relu")
    check_backward(0, 5, 4, types, "relu")
    check_backward(0, 500, 300, types, "none", accumulate=True)
    check_backward(0, 5, 4, types, "relu", want=("x",))
    torch.cuda.synchronize()


def test_residual_layer_in_place():
    """x as its own residual; the residual's buffer as the result; grad_y as what is added to the gradient of x."""
    import torch
    for R, D in ((50, 64), (1500, 512)):
        d = inputs(R, D, D, ("fp32", "fp32"))
        f = torch.float32
        cfg = bd.make_dense_config(R, D, D, activation=bd.ACT_RELU)
        x, W, b = put(d["x"], f), put(d["W"], f), put(d["bias"], f)
        y, z, ws = torch.empty(R, D, device="cuda:0"), torch.empty(R, D, device="cuda:0"), workspace(cfg)
        bd.spcfg_dense_forward(cfg, x, W, b, x, y, z, ws)
        r = put(d["x"], f)
        bd.spcfg_dense_forward(cfg, x, W, b, r, r, None, ws)
        assert torch.equal(r, y)
        want, wz = NO.forward(d["x"], d["W"], d["bias"], d["x"], "relu")
        close("y", values(y), want, product_tol(d["x"], d["W"]) + 2.0 ** -20 * (1 + np.abs(want) + np.abs(wz)))
        gy, gx = put(d["grad_y"], f), torch.empty(R, D, device="cuda:0")
        bd.spcfg_dense_backward(cfg, x, W, z, gy, gy, gx, None, None, ws)
        a = put(d["grad_y"], f)
        bd.spcfg_dense_backward(cfg, x, W, z, gy, a, a, None, None, ws)  # the added tensor's buffer as the result
        assert torch.equal(a, gx)


@pytest.mark.parametrize("R,I,O", [(40, 100, 50), (700, 700, 900), (300, 4500, 400)])
def test_fp32_rows_of_any_scale(R, I, O):
    """Rows of x and W that are fifteen orders of magnitude apart, and values eight orders apart inside each: every result is as
    exact as its own terms allow.  An infinite value makes its row NaN and no other."""
    import torch
    rng = np.random.default_rng(R)
    spread = lambda n, m: rng.normal(size=(n, m)) * 10.0 ** rng.uniform(-8, 0, size=(n, m)) * 10.0 ** rng.uniform(-15, 15, size=(n, 1))
    x, W = rounded(spread(R, I), False), rounded(spread(O, I), False)
    x[3] = 0.0
    cfg = bd.make_dense_config(R, I, O)
    f = torch.float32
    y, ws = torch.empty(R, O, device="cuda:0"), workspace(cfg)
    tx, tW = put(x, f), put(W, f)
    bd.spcfg_dense_forward(cfg, tx, tW, None, None, y, None, ws)
    want = x @ W.T
    close("y", values(y), want, product_tol(x, W) + 2.0 ** -24 * np.abs(want) + 2.0 ** -126)
    tx[5, 7] = float("inf")
    bd.spcfg_dense_forward(cfg, tx, tW, None, None, y, None, ws)
    got = values(y)
    assert np.all(np.isnan(got[5]))
    rest = np.arange(R) != 5
    close("other rows", got[rest], want[rest], (product_tol(x, W) + 2.0 ** -24 * np.abs(want) + 2.0 ** -126)[rest])


def test_activations_of_extreme_values():
    """Infinite and huge sums reach the activation as they are (bf16 operands); slopes there are 0 or 1; NaN stays NaN."""
    import torch
    b16 = torch.bfloat16
    x = torch.tensor([[float("inf")], [float("-inf")], [100.0], [-100.0], [float("nan")], [0.0]], dtype=b16, device="cuda:0")
    W = torch.ones(1, 1, dtype=b16, device="cuda:0")
    inf, nan = float("inf"), float("nan")
    for act, want, slope in (("relu", [inf, 0, 100, 0, nan, 0], [1, 0, 1, 0, nan, 0]),
                             ("gelu", [inf, 0, 100, 0, nan, 0], [1, 0, 1, 0, nan, 0.5]),
                             ("silu", [inf, 0, 100, -100 * np.exp(-100.0), nan, 0], [1, 0, 1, 0, nan, 0.5])):
        cfg = bd.make_dense_config(6, 1, 1, bd.TYPE_BF16, bd.TYPE_F32, ACTS[act])
        y, z = torch.empty(6, 1, device="cuda:0"), torch.empty(6, 1, device="cuda:0")
        bd.spcfg_dense_forward(cfg, x, W, None, None, y, z, workspace(cfg))
        assert np.allclose(values(y)[:, 0], want, rtol=1e-6, atol=1e-30, equal_nan=True), (act, values(y))
        gx = torch.empty(6, 1, dtype=b16, device="cuda:0")
        bd.spcfg_dense_backward(cfg, x, W, z, torch.ones(6, 1, device="cuda:0"), None, gx, None, None, workspace(cfg))
        assert np.allclose(values(gx)[:, 0], slope, atol=1e-6, equal_nan=True), (act, values(gx))


@pytest.mark.parametrize("R,I,O", [(100, 64, 200), (1300, 512, 1100)])
def test_streams_and_graphs(R, I, O):
    """On a stream of the caller's, and captured: two graphs share a workspace, are replayed in turns between eager calls on it,
    and give what the eager calls gave, bit by bit, also on new inputs."""
    import torch
    d = inputs(R, I, O, ("fp32", "fp32"))
    f = torch.float32
    cfg = bd.make_dense_config(R, I, O, activation=bd.ACT_SILU)
    x, W, b, gy = (put(d[k], f) for k in ("x", "W", "bias", "grad_y"))
    e = lambda *s: torch.empty(*s, device="cuda:0")
    y, z, gx, gW, gb, ws = e(R, O), e(R, O), e(R, I), e(O, I), e(O), workspace(cfg)

    def fwd():
        bd.spcfg_dense_forward(cfg, x, W, b, None, y, z, ws)

    def bwd():
        bd.spcfg_dense_backward(cfg, x, W, z, gy, None, gx, gW, gb, ws)
    outs = (y, z, gx, gW, gb)
    fwd()
    bwd()
    torch.cuda.synchronize()
    eager = [t.clone() for t in outs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for t in outs:
        t.fill_(float("nan"))
    with torch.cuda.stream(side):
        side.wait_stream(torch.cuda.default_stream())
        fwd()
        bwd()
    side.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(outs, eager))
    graphs = []
    for step in (fwd, bwd):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
        graphs.append(g)
    for turn in range(3):
        x.mul_(1.0 if turn == 0 else 0.5)
        for t in outs:
            t.fill_(float("nan"))
        graphs[0].replay()
        graphs[1].replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        fwd()
        bwd()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(outs, got)), turn


def test_matrices_of_more_than_32_bits_of_bytes():
    """y, z and grad_y of 4.6 GB each: the last rows, and gradients that all rows add up to; references in 64 bits on the GPU."""
    import torch
    R, I, O = 140001, 64, 16392
    print("case dense far offsets", R, I, O, flush=True)
    b16, dev = torch.bfloat16, "cuda:0"
    g = torch.Generator(device=dev)
    g.manual_seed(3)
    n = lambda *s: torch.randn(*s, generator=g, device=dev)
    x, W, b = n(R, I).to(b16), (0.2 * n(O, I)).to(b16), n(O).to(b16)
    cfg = bd.make_dense_config(R, I, O, bd.TYPE_BF16, bd.TYPE_BF16, bd.ACT_RELU)
    ws = workspace(cfg)
    y, z = torch.empty(R, O, dtype=b16, device=dev), torch.empty(R, O, dtype=b16, device=dev)
    bd.spcfg_dense_forward(cfg, x, W, b, None, y, z, ws)
    D = lambda t: t.double()
    rows = torch.cat([torch.arange(3), torch.arange(R // 2, R // 2 + 3), torch.arange(R - 5, R)]).to(dev)
    want = D(x[rows]) @ D(W).t() + D(b)
    q = torch.sqrt((D(x[rows]) ** 2) @ (D(W) ** 2).t())
    tol = U * (16 + 6 * I / 16) * 2 * q + (2.0 ** -8 + 2.0 ** -20) * want.abs() + 2.0 ** -20
    close("preact", values(z[rows]), want.cpu().numpy(), tol.cpu().numpy())
    close("y", values(y[rows]), want.clamp(min=0).cpu().numpy(), tol.cpu().numpy())
    gy = y  # (its own buffer as an upstream gradient: any values do)
    gx, gW, gb = torch.empty(R, I, dtype=b16, device=dev), torch.empty(O, I, dtype=b16, device=dev), torch.empty(O, dtype=b16, device=dev)
    bd.spcfg_dense_backward(cfg, x, W, z, gy, None, gx, gW, gb, ws)
    cols = torch.tensor([0, 1, O // 2, O - 2, O - 1], device=dev)
    for name, got, A, B, K in (("grad_x", gx[rows], D(gy[rows]) * (D(z[rows]) > 0), D(W), O),
                               ("grad_W", gW[cols], (D(gy[:, cols]) * (D(z[:, cols]) > 0)).t(), D(x), R)):
        want, q = A @ B, torch.sqrt((A ** 2) @ (B ** 2))
        tol = (U * (16 + 6 * K / 16) * 2 + 4 * 2.0 ** -8) * q + (2.0 ** -8 + 2.0 ** -22) * want.abs()
        close(name, values(got), want.cpu().numpy(), tol.cpu().numpy())
    want = (D(gy[:, cols]) * (D(z[:, cols]) > 0)).sum(0)
    # (terms of one sign: every addition rounds a sum as large as the result, 16 rows in a row, then parts of the rows)
    close("grad_bias", values(gb[cols]), want.cpu().numpy(), ((2.0 ** -8 + 2.0 ** -15) * want.abs()).cpu().numpy())


def test_the_binding_refuses_other_tensors():
    import torch
    e = lambda *s, **k: torch.empty(*s, device="cuda:0", **k)
    cfg = bd.make_dense_config(4, 8, 6)
    ok = dict(x=e(4, 8), W=e(6, 8), bias=e(6), residual=None, y=e(4, 6), preact=None, workspace=None)
    for bad, what in ((dict(x=e(4, 7)), ValueError), (dict(W=e(8, 6).t()), TypeError), (dict(bias=e(6, dtype=torch.float64)), TypeError),
                      (dict(y=torch.empty(4, 6)), TypeError), (dict(residual=e(4, 8)), ValueError), (dict(x=[1.0]), TypeError),
                      (dict(workspace=e(64)), TypeError)):
        with pytest.raises(what):
            bd.spcfg_dense_forward(cfg, **{**ok, **bad})
    with pytest.raises(bd.SpcfgError) as err:
        bd.spcfg_dense_forward(bd.make_dense_config(4, 8, 6, 5, 0), **ok)
    assert err.value.code == -5
    big = bd.make_dense_config(2048, 512, 2048)
    with pytest.raises(bd.SpcfgError) as err:
        bd.spcfg_dense_forward(big, e(2048, 512), e(2048, 512), None, None, e(2048, 2048), None, None)
    assert err.value.code == -1


@pytest.mark.parametrize("types", TYPES, ids="-".join)
@pytest.mark.parametrize("R,I,O", [(8000, 5, 2000), (2500, 641, 1003), (1500, 1028, 774), (2200, 513, 1021)])
def test_rows_of_odd_lengths_on_tiles(R, I, O, types):
    """Ends of rows at every place of eight values, rows shorter than eight, and the same from an address that nothing lies on."""
    for shift in (0, 1):
        print("case dense odd", R, I, O, types, shift, flush=True)
        check_forward(R, I, O, types, "silu", shift=shift)
        check_backward(R, I, O, types, "silu", shift=shift)
