"""GPU tests of the gradients of bf16 layers to what their own rounding leaves: dz = grad_y * act'(z) is held in 32 bits and enters
the products as two bf16 pieces, so that the gradients are as good as those of a 32-bit dz.

Tolerances, per element, as in test_gpu_dense.py but for dz: the product's own sums, 2^-23 (16 + 12 K / 16) 2 q with two piece products
a step, q the root of the terms' squares; slopes 2^-21 (1 + |z|) of grad_y and the pieces 2^-17 of dz, terms of random signs, 4 times
their root sum of squares; half a step of the result, 2^-8 of it.  One rounding of dz to bf16, 2^-8 of each term, does not fit: where a
gradient is a tenth of q or less (one in twelve) its half step is a tenth of that.
"""
import numpy as np
import pytest

from oracle import network_oracle as NO
from operator_util import close, guarded, put, rounded, values
from paper_2310_14997_amd import binding as bd
from test_gpu_dense import ACTS, U, d_of, inputs, t_of, workspace

pytestmark = pytest.mark.gpu


def check(R, I, O, out_type, act, shift=0):
    types = ("bf16", out_type)
    d = inputs(R, I, O, types, seed=2)
    ti, to = d_of("bf16"), d_of(out_type)
    z = rounded(d["x"] @ d["W"].T + d["bias"], out_type == "bf16")
    cfg = bd.make_dense_config(R, I, O, t_of("bf16"), t_of(out_type), ACTS[act])
    gx, x_ok = guarded((R, I), ti, shift)
    gW, W_ok = guarded((O, I), ti, shift)
    gb, b_ok = guarded((O,), ti, shift)
    bd.spcfg_dense_backward(cfg, put(d["x"], ti, shift), put(d["W"], ti, shift), put(z, to, shift) if act != "none" else None,
                            put(d["grad_y"], to, shift), None, gx, gW, gb, workspace(cfg))
    wx, wW, wb = NO.backward(d["x"], d["W"], z, d["grad_y"], act)
    dz = d["grad_y"] * NO.act_slope(z, act)
    off = 2.0 ** -17 * np.abs(dz) + 2.0 ** -21 * np.abs(d["grad_y"]) * (1 + np.abs(z)) * (act in ("gelu", "silu"))

    def tol(A, E, B, want):
        K, sq = A.shape[1], lambda a, b: np.sqrt((a * a) @ (b * b))
        return U * (16 + 12 * K / 16) * 2 * sq(A, B) + 4 * sq(E, B) + (2.0 ** -8 + 2.0 ** -22) * np.abs(want)
    close("grad_x", values(gx), wx, tol(dz, off, d["W"], wx))
    close("grad_W", values(gW), wW, tol(dz.T, off.T, d["x"], wW))
    close("grad_bias", values(gb), wb, tol(dz.T, off.T, np.ones((R, 1)), wb[:, None])[:, 0])
    for ok in (x_ok, W_ok, b_ok):
        ok()


# products in registers on tiles of 16 and 32, on tiles in LDS of 64 and 128, whole and ragged
SIZES = [(3, 64, 32), (70, 64, 96), (129, 48, 1000), (300, 520, 264), (1025, 264, 1111), (130, 2050, 700), (2048, 512, 512),
         (777, 333, 1999), (4100, 72, 130), (8200, 512, 520)]


@pytest.mark.parametrize("out_type,act", [("fp32", "none"), ("fp32", "relu"), ("fp32", "silu"), ("bf16", "gelu"), ("bf16", "relu")])
@pytest.mark.parametrize("R,I,O", SIZES)
def test_gradients_as_of_a_32_bit_dz(R, I, O, out_type, act):
    print("case dense pieces", R, I, O, out_type, act, flush=True)
    check(R, I, O, out_type, act)
    if R in (70, 1025):
        check(R, I, O, out_type, act, shift=1)


@pytest.mark.parametrize("out_type,act", [("fp32", "none"), ("bf16", "silu")])
def test_wide(out_type, act):
    """Tiles of 256; the reference is 64-bit arithmetic on the GPU, over a sample of rows and columns."""
    import torch
    R, I, O = 4100, 4104, 4112
    print("case dense pieces wide", out_type, act, flush=True)
    g = torch.Generator(device="cuda:0")
    g.manual_seed(9)
    n = lambda *s: torch.randn(*s, generator=g, device="cuda:0")
    b16, to = torch.bfloat16, d_of(out_type)
    x, W, gy, z = n(R, I).to(b16), (0.02 * n(O, I)).to(b16), n(R, O).to(to), n(R, O).to(to)
    cfg = bd.make_dense_config(R, I, O, bd.TYPE_BF16, t_of(out_type), ACTS[act])
    gx, gW = torch.empty(R, I, dtype=b16, device="cuda:0"), torch.empty(O, I, dtype=b16, device="cuda:0")
    bd.spcfg_dense_backward(cfg, x, W, None if act == "none" else z, gy, None, gx, gW, None, workspace(cfg))
    D = lambda t: t.double()
    s = torch.sigmoid(D(z))
    dz = D(gy) if act == "none" else D(gy) * (s + D(z) * s * (1 - s))
    off = 2.0 ** -17 * dz.abs() + (0.0 if act == "none" else 2.0 ** -21 * D(gy).abs() * (1 + D(z).abs()))
    rows = torch.cat([torch.arange(0, R, 41), torch.arange(R - 5, R)]).cuda()
    cols = torch.cat([torch.arange(0, O, 37), torch.arange(O - 5, O)]).cuda()
    for name, got, A, E, B, K in (("grad_x", gx[rows], dz[rows], off[rows], D(W), O),
                                  ("grad_W", gW[cols], dz[:, cols].t().contiguous(), off[:, cols].t().contiguous(), D(x), R)):
        want = A @ B
        tol = U * (16 + 12 * K / 16) * 2 * torch.sqrt((A ** 2) @ (B ** 2)) + 4 * torch.sqrt((E ** 2) @ (B ** 2)) \
            + (2.0 ** -8 + 2.0 ** -22) * want.abs()
        close(name, values(got), want.cpu().numpy(), tol.cpu().numpy())


def test_infinite_gradients_stay_in_their_rows():
    """An infinite grad_y makes its row of grad_x and its column's grad_W infinite or NaN, and no other value."""
    import torch
    b16, f = torch.bfloat16, torch.float32
    for R, I, O in ((40, 64, 48), (2048, 512, 512)):
        d = inputs(R, I, O, ("bf16", "fp32"), seed=3)
        cfg = bd.make_dense_config(R, I, O, bd.TYPE_BF16, bd.TYPE_F32)
        x, W, gy = put(d["x"], b16), put(d["W"], b16), put(d["grad_y"], f)
        e = lambda *s: torch.empty(*s, dtype=b16, device="cuda:0")
        outs = [(e(R, I), e(O, I), e(O)) for _ in range(2)]
        for k, (gx, gW, gb) in enumerate(outs):
            if k:
                gy[7, 5] = float("inf")
            bd.spcfg_dense_backward(cfg, x, W, None, gy, None, gx, gW, gb, workspace(cfg))
        (ax, aW, ab), (bx, bW, bb) = outs
        assert not bool(torch.isfinite(bx[7]).any()) and not bool(torch.isfinite(bW[5]).any()) and float(bb[5]) == float("inf")
        rest = torch.arange(R, device="cuda:0") != 7
        assert torch.equal(ax[rest], bx[rest])
        rest = torch.arange(O, device="cuda:0") != 5
        assert torch.equal(aW[rest], bW[rest]) and torch.equal(ab[rest], bb[rest])
