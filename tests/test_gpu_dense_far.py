"""GPU tests of layers of very many rows and of very long rows: sizes from 2^22 on, results of 2^33 values (more than one launch's
threads where a workgroup takes a tile of 32 x 32), and sums of millions of terms of one sign.

Tolerances: random data as in test_gpu_dense.py; sums of equal terms by the additions one behind the other, each off by at most 2^-24 of
the sum so far, named at the test."""
import numpy as np
import pytest

from operator_util import close, values
from paper_2310_14997_amd import binding as bd
from test_gpu_dense import TYPES, U, d_of, half_step, t_of, workspace

pytestmark = pytest.mark.gpu
MANY = (1 << 22) + 37


@pytest.mark.parametrize("types", TYPES, ids="-".join)
def test_sums_of_equal_terms_over_many_rows(types):
    """The bias's gradient: runs of 128 additions of four rows' sums, some 2050 such sums in 8 or 4 wavefronts and eight sums each, at most
    65 one behind the other, and 15 to join: fewer than 300.  The gradient of W: at most 2^12 matrix instructions of each piece product
    in a row (each taken as two roundings), six, two or one of them, then 65 parts."""
    import torch
    R, I, O = MANY, 8, 24
    print("case dense many equal rows", types, flush=True)
    ti, to = d_of(types[0]), d_of(types[1])
    x, W = torch.full((R, I), 0.1, dtype=ti, device="cuda:0"), torch.full((O, I), 0.3, dtype=ti, device="cuda:0")
    gy = torch.full((R, O), 0.1, dtype=to, device="cuda:0")
    cfg = bd.make_dense_config(R, I, O, t_of(types[0]), t_of(types[1]))
    gx, gW, gb = torch.empty_like(x), torch.empty_like(W), torch.empty(O, dtype=ti, device="cuda:0")
    bd.spcfg_dense_backward(cfg, x, W, None, gy, None, gx, gW, gb, workspace(cfg))
    v = lambda t: float(t.flatten()[0].double())
    hs = half_step(types[0])
    close("grad_bias", values(gb), np.full(O, R * v(gy)), R * v(gy) * (300 * 2.0 ** -24 + hs))
    pieces = 6 if types[0] == "fp32" else 2 if types[1] == "fp32" else 1
    close("grad_W", values(gW), np.full((O, I), R * v(gy) * v(x)), R * v(gy) * v(x) * ((2 * 2 ** 12 * pieces + 100) * 2.0 ** -24 + hs))
    close("grad_x", values(gx[-3:]), np.full((3, I), O * v(gy) * v(W)), O * v(gy) * v(W) * (2.0 ** -17 + hs))


def test_long_rows_of_equal_terms():
    """Rows of 2^22 inputs, products in registers: 256 chunks of six piece products one behind the other, then 64 runs and 8 wavefronts."""
    import torch
    R, I, O = 3, (1 << 22) + 8, 5
    print("case dense long equal rows", flush=True)
    x, W = torch.full((R, I), 0.1, device="cuda:0"), torch.full((O, I), 0.1, device="cuda:0")
    cfg = bd.make_dense_config(R, I, O)
    y = torch.empty(R, O, device="cuda:0")
    bd.spcfg_dense_forward(cfg, x, W, None, None, y, None, workspace(cfg))
    want = I * float(x[0, 0].double()) ** 2
    close("y", values(y), np.full((R, O), want), want * (256 * 6 + 64 + 8 + 2) * 2.0 ** -24)


@pytest.mark.parametrize("types", TYPES, ids="-".join)
@pytest.mark.parametrize("R,I,O", [(MANY, 24, 40), (MANY, 33, 7), (2051, 16, (1 << 22) + 9), (70, (1 << 22) + 11, 9)])
def test_far_sizes(R, I, O, types):
    """All results of samples of rows and columns, the last ones among them; references in 64 bits on the GPU."""
    import torch
    print("case dense far", R, I, O, types, flush=True)
    if O > MANY - 64 and types[1] == "fp32":
        R = 131  # (R x O values of 4 bytes stay small)
    g = torch.Generator(device="cuda:0")
    g.manual_seed(5)
    ti, to = d_of(types[0]), d_of(types[1])
    n = lambda t, *s: torch.randn(*s, generator=g, device="cuda:0").to(t) if s[0] * s[-1] < 1 << 30 else \
        torch.cat([torch.randn(min(64, s[0] - i), *s[1:], generator=g, device="cuda:0").to(t) for i in range(0, s[0], 64)])
    x, W, b = n(ti, R, I), n(ti, O, I), n(ti, O)
    cfg = bd.make_dense_config(R, I, O, t_of(types[0]), t_of(types[1]), bd.ACT_RELU)
    y, z, ws = torch.empty(R, O, dtype=to, device="cuda:0"), torch.empty(R, O, dtype=to, device="cuda:0"), workspace(cfg)
    bd.spcfg_dense_forward(cfg, x, W, b, None, y, z, ws)
    D = lambda t: t.double()
    ends = lambda k: torch.unique(torch.tensor([0, 1, k // 3, k // 2, k - 2, k - 1], device="cuda:0").clamp(0, k - 1))
    rows, cols = ends(R), ends(O)
    want = D(x[rows]) @ D(W[cols]).t().contiguous() + D(b[cols])
    q = torch.sqrt((D(x[rows]) ** 2) @ (D(W[cols]) ** 2).t().contiguous())
    tol = U * (16 + 6 * I / 16) * 2 * q + 2.0 ** -20 * (want.abs() + D(b[cols]).abs()) + half_step(types[1]) * want.abs()
    close("preact", values(z[rows][:, cols]), want.cpu().numpy(), tol.cpu().numpy())
    close("y", values(y[rows][:, cols]), want.clamp(min=0).cpu().numpy(), tol.cpu().numpy())
    gy = n(to, R, O)
    gx, gW, gb = torch.empty_like(x), torch.empty_like(W), torch.empty_like(b)
    bd.spcfg_dense_backward(cfg, x, W, z, gy, None, gx, gW, gb, ws)
    lossy = 4 * 2.0 ** -17 if types[0] == "bf16" else 0.0
    ins = ends(I)
    for name, got, A, B, K in (("grad_x", gx[rows][:, ins], D(gy[rows]) * (z[rows] > 0), D(W[:, ins]), O),
                               ("grad_W", gW[cols][:, ins], (D(gy[:, cols]) * (z[:, cols] > 0)).t().contiguous(), D(x[:, ins]), R)):
        want, q = A @ B, torch.sqrt((A ** 2) @ (B ** 2))
        tol = (U * (16 + 12 * K / 16) * 2 + lossy) * q + (half_step(types[0]) + 2.0 ** -22) * want.abs()
        close(name, values(got), want.cpu().numpy(), tol.cpu().numpy())
    dz = D(gy[:, cols]) * (z[:, cols] > 0)
    want, q = dz.sum(0), torch.sqrt((dz ** 2).sum(0))
    close("grad_bias", values(gb[cols]), want.cpu().numpy(),
          (U * (16 + 6 * R / 16) * 2 * q + (half_step(types[0]) + 2.0 ** -22) * want.abs()).cpu().numpy())


@pytest.mark.parametrize("R,I,O", [((1 << 22) + 64, 8, 2056), (2080, 8, (1 << 22) + 8)])
def test_results_of_more_than_one_launch(R, I, O):
    """More than 2^33 results: y alone has 17 GB."""
    import torch
    print("case dense launches", R, I, O, flush=True)
    b16 = torch.bfloat16
    g = torch.Generator(device="cuda:0")
    g.manual_seed(6)
    x, W = (torch.randn(k, I, generator=g, device="cuda:0").to(b16) for k in (R, O))
    cfg = bd.make_dense_config(R, I, O, bd.TYPE_BF16, bd.TYPE_BF16)
    y, ws = torch.full((R, O), 7.0, dtype=b16, device="cuda:0"), workspace(cfg)
    bd.spcfg_dense_forward(cfg, x, W, None, None, y, None, ws)
    rows, cols = torch.arange(0, R, max(1, R // 300), device="cuda:0"), torch.arange(0, O, max(1, O // 300), device="cuda:0")
    rows[-1], cols[-1] = R - 1, O - 1
    want = x[rows].double() @ W[cols].double().t().contiguous()
    q = torch.sqrt((x[rows].double() ** 2) @ (W[cols].double() ** 2).t().contiguous())
    close("y", values(y[rows][:, cols]), want.cpu().numpy(), (U * 40 * q + 2.0 ** -8 * want.abs()).cpu().numpy())
    # and back, from y's own buffer: any values do
    gx, gW = torch.empty_like(x), torch.empty_like(W)
    bd.spcfg_dense_backward(cfg, x, W, None, y, None, gx, gW, None, ws)
    rows, cols = rows[-3:], cols[-3:]
    for name, got, A, B, K in (("grad_x", gx[rows], y[rows].double(), W.double(), O),
                               ("grad_W", gW[cols], y[:, cols].double().t().contiguous(), x.double(), R)):
        want, size = A @ B, A.abs() @ B.abs()
        close(name, values(got), want.cpu().numpy(), (U * 2 ** 13 * size + 2.0 ** -8 * want.abs()).cpu().numpy())
