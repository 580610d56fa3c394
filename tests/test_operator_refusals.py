"""What the layers and losses refuse, on the host and before anything is launched: every call here is made with pointers
that are no memory at all."""
import ctypes as C

import pytest

from paper_2310_14997_amd import binding as bd

P = [0x10000000 * (i + 1) for i in range(12)]  # far apart, on 256 bytes
ARG, SHAPE, WORKSPACE, UNSUPPORTED = -1, -2, -4, -5


def dense(rows=4, n_in=8, n_out=8, ti=0, to=0, act=1, flags=0, size=None):
    cfg = bd.make_dense_config(rows, n_in, n_out, ti, to, act, flags)
    if size is not None:
        cfg.struct_size = size
    return cfg


def forward(cfg, x=P[0], W=P[1], bias=P[2], residual=P[3], y=P[4], preact=P[5], ws=P[10], nbytes=1 << 40):
    return bd.load().spcfg_dense_forward(C.byref(cfg), x, W, bias, residual, y, preact, ws, nbytes, None)


def backward(cfg, x=P[0], W=P[1], preact=P[2], gy=P[3], add=P[4], gx=P[5], gW=P[6], gb=P[7], ws=P[10], nbytes=1 << 40):
    return bd.load().spcfg_dense_backward(C.byref(cfg), x, W, preact, gy, add, gx, gW, gb, ws, nbytes, None)


@pytest.mark.parametrize("kw,code", [
    (dict(rows=-1), SHAPE), (dict(n_in=0), SHAPE), (dict(n_out=0), SHAPE), (dict(rows=(1 << 24) + 1), SHAPE),
    (dict(rows=1 << 24, n_in=1 << 13), SHAPE), (dict(n_in=1 << 20, n_out=1 << 17), SHAPE),
    (dict(ti=0, to=1), UNSUPPORTED), (dict(ti=2), UNSUPPORTED), (dict(ti=1, to=2), UNSUPPORTED), (dict(act=4), UNSUPPORTED),
    (dict(act=-1), UNSUPPORTED), (dict(flags=2), UNSUPPORTED), (dict(size=4), ARG),
], ids=str)
def test_layers_refuse_configurations(kw, code):
    cfg = dense(**kw)
    assert forward(cfg) == code and backward(cfg) == code
    assert bd.load().spcfg_dense_workspace_bytes(C.byref(cfg), C.byref(C.c_size_t())) == code


def test_layers_refuse_missing_misaligned_and_shared_memory():
    assert bd.load().spcfg_dense_workspace_bytes(C.byref(dense()), None) == ARG
    for kw in (dict(x=None), dict(W=None), dict(y=None), dict(x=P[0] + 2), dict(y=P[4] + 1), dict(y=P[0]), dict(y=P[1] + 4),
               dict(preact=P[4]), dict(preact=P[4] + 64), dict(preact=P[0]), dict(preact=P[3]), dict(y=P[3] + 4),
               dict(y=P[2])):
        assert forward(dense(), **kw) == ARG, kw
    for kw in (dict(x=None), dict(W=None), dict(gy=None), dict(preact=None), dict(gx=None, gW=None, gb=None), dict(gW=None),
               dict(gx=None), dict(gx=P[3]), dict(gx=P[0]), dict(gW=P[1]), dict(gW=P[5]), dict(gb=P[6] + 32), dict(gx=P[2]),
               dict(add=P[3], gx=P[3]), dict(gx=P[4] + 4), dict(gb=P[7] + 1), dict(gW=P[4])):
        assert backward(dense(), **kw) == ARG, kw


def test_layers_refuse_workspaces():
    cfg = dense(rows=4096, n_in=520, n_out=1000)
    n = C.c_size_t()
    assert bd.load().spcfg_dense_workspace_bytes(C.byref(cfg), C.byref(n)) == 0
    if n.value:
        for call in (forward, backward):
            assert call(cfg, ws=None) == ARG
            assert call(cfg, ws=P[10] + 16) == WORKSPACE
            assert call(cfg, nbytes=n.value - 1) == WORKSPACE


def distill(which, type=0, rows=3, V=50, k=4, s=P[0], t=P[1], ids=P[2], tau=1.0, gl=P[3], loss=P[4], lse=P[5], g=P[6],
            ws=P[10], nbytes=1 << 40):
    lib = bd.load()
    if which == "forward":
        return lib.spcfg_distill_forward(type, rows, V, k, s, t, ids, tau, loss, lse, ws, nbytes, None)
    if which == "backward":
        return lib.spcfg_distill_backward(type, rows, V, k, s, t, ids, tau, lse, gl, g, None)
    return lib.spcfg_distill_forward_backward(type, rows, V, k, s, t, ids, tau, gl, loss, lse, g, ws, nbytes, None)


@pytest.mark.parametrize("which", ["forward", "backward", "both"])
def test_distillation_refuses(which):
    for kw, code in ((dict(type=2), UNSUPPORTED), (dict(rows=-1), SHAPE), (dict(V=0), SHAPE), (dict(k=0), SHAPE),
                     (dict(k=1025), SHAPE), (dict(rows=1 << 20, V=1 << 17), SHAPE), (dict(V=(1 << 24) + 1), SHAPE),
                     (dict(tau=0.0), ARG), (dict(tau=-1.0), ARG), (dict(tau=float("nan")), ARG), (dict(tau=float("inf")), ARG),
                     (dict(tau=1e-40), ARG), (dict(s=None), ARG), (dict(t=None), ARG), (dict(ids=None), ARG),
                     (dict(lse=None), ARG), (dict(s=P[0] + 2), ARG), (dict(ids=P[2] + 2), ARG), (dict(type=1, t=P[1] + 1), ARG)):
        assert distill(which, **kw) == code, kw
    if which != "backward":
        assert distill(which, loss=None) == ARG
        for kw, code in ((dict(ws=None), ARG), (dict(ws=P[10] + 8), WORKSPACE), (dict(nbytes=8), WORKSPACE)):
            assert distill(which, V=200000, **kw) == code
    if which != "forward":
        for kw in (dict(g=None), dict(g=P[0]), dict(g=P[0] + 4), dict(g=P[1]), dict(g=P[2]), dict(g=P[3]), dict(g=P[6] + 1)):
            assert distill(which, **kw) == ARG, kw


def test_distillation_workspaces():
    assert bd.spcfg_distill_workspace_bytes(2048, 10000) == 0 and bd.spcfg_distill_workspace_bytes(0, 1 << 24) == 0
    assert bd.spcfg_distill_workspace_bytes(8, 131071) > 0
    for rows, V in ((-1, 5), (5, 0)):
        with pytest.raises(bd.SpcfgError) as e:
            bd.spcfg_distill_workspace_bytes(rows, V)
        assert e.value.code == SHAPE
    assert bd.load().spcfg_distill_workspace_bytes(4, 4, None) == ARG


def preference(which, B=6, n=4, z=P[0], ref=P[1], c=P[2], r=P[3], beta=0.1, eps=0.0, gl=P[4], loss=P[5], margin=P[6], g=P[7]):
    lib = bd.load()
    if which == "forward":
        return lib.spcfg_preference_forward(B, n, z, ref, c, r, beta, eps, loss, margin, None)
    if which == "backward":
        return lib.spcfg_preference_backward(B, n, z, ref, c, r, beta, eps, gl, g, None)
    return lib.spcfg_preference_forward_backward(B, n, z, ref, c, r, beta, eps, gl, loss, margin, g, None)


@pytest.mark.parametrize("which", ["forward", "backward", "both"])
def test_preference_refuses(which):
    nan = float("nan")
    for kw, code in ((dict(B=0), SHAPE), (dict(B=65537), SHAPE), (dict(n=-1), SHAPE), (dict(n=(1 << 20) + 1), SHAPE),
                     (dict(beta=0.0), ARG), (dict(beta=nan), ARG), (dict(beta=float("inf")), ARG), (dict(eps=-0.1), ARG),
                     (dict(eps=1.1), ARG), (dict(eps=nan), ARG), (dict(z=None), ARG), (dict(c=None), ARG), (dict(r=None), ARG)):
        assert preference(which, **kw) == code, kw
    if which != "backward":
        for kw in (dict(loss=None), dict(margin=None), dict(loss=P[0] + 4), dict(margin=P[5] + 8), dict(loss=P[2])):
            assert preference(which, **kw) == ARG, kw
    if which != "forward":
        for kw in (dict(g=None), dict(g=P[0]), dict(g=P[3] + 4), dict(g=P[4])):
            assert preference(which, **kw) == ARG, kw


def test_the_binding_refuses_host_tensors():
    import torch
    z = torch.zeros(4)
    i = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(TypeError):
        bd.spcfg_preference_forward(z, None, i, i, 0.1, 0.0, torch.zeros(2), torch.zeros(2))
    with pytest.raises(TypeError):
        bd.spcfg_distill_forward(torch.zeros(2, 5), torch.zeros(2, 3), torch.zeros(2, 3, dtype=torch.int32), 1.0,
                                 torch.zeros(2), torch.zeros(2), None)
    with pytest.raises(TypeError):
        bd.spcfg_distill_forward(torch.zeros(2, 5, dtype=torch.float64), None, torch.zeros(2, 3), 1.0, None, None, None)
    with pytest.raises(TypeError):
        bd.spcfg_dense_forward(dense(), torch.zeros(4, 8), torch.zeros(8, 8), None, None, torch.zeros(4, 8), None, None)


@pytest.mark.parametrize("which", ["forward", "backward", "both"])
def test_temperatures_without_a_finite_inverse(which):
    """What the scores are multiplied by, log2(e) / temperature, has to be a finite float."""
    assert distill(which, tau=4e-39) == ARG
    assert distill(which, tau=0.0) == ARG
