"""Memory that the layers and losses refuse on the host: outputs and workspaces that share it with anything else, part of it or all.
Every call is made with pointers that are no memory at all."""
import ctypes as C

import pytest

from paper_2310_14997_amd import binding as bd
from test_operator_refusals import ARG, P, backward, dense, distill, forward, preference

LONG = 200000  # a row that takes a workspace


def test_workspaces_of_layers():
    cfg = dense(rows=4096, n_in=520, n_out=1000)
    n = C.c_size_t()
    assert bd.load().spcfg_dense_workspace_bytes(C.byref(cfg), C.byref(n)) == 0 and 0 < n.value < P[0]
    for i in range(6):
        assert forward(cfg, ws=P[i]) == ARG, i
    for i in range(8):
        assert backward(cfg, ws=P[i]) == ARG, i
    assert forward(cfg, ws=P[0] + 4096) == ARG and backward(cfg, ws=P[6] - (n.value - 256) // 256 * 256) == ARG


@pytest.mark.parametrize("which", ["forward", "both"])
def test_outputs_of_the_distillation(which):
    for kw in (dict(loss=P[5]), dict(loss=P[5] + 8), dict(loss=P[0]), dict(lse=P[0] + 40), dict(loss=P[1]), dict(lse=P[2] + 4)):
        assert distill(which, **kw) == ARG, kw
    if which == "both":
        for kw in (dict(loss=P[3]), dict(lse=P[3] + 8), dict(loss=P[6]), dict(lse=P[6] + 196), dict(g=P[5] + 4), dict(g=P[4] - 4)):
            assert distill(which, **kw) == ARG, kw
    for i in range(3 if which == "forward" else 7):
        assert distill(which, V=LONG, ws=P[i]) == ARG, i


def test_gradients_alone_beside_their_inputs():
    for kw in (dict(g=P[0]), dict(g=P[1]), dict(g=P[2]), dict(g=P[3]), dict(g=P[5]), dict(g=P[5] + 8)):
        assert distill("backward", **kw) == ARG, kw


def test_preferences():
    for kw in (dict(loss=P[6]), dict(loss=P[6] + 12), dict(g=P[5]), dict(g=P[6] - 20), dict(margin=P[1] + 20)):
        assert preference("both", **kw) == ARG, kw
