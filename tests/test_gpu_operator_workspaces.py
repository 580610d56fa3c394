"""GPU tests of the layers' and the distillation's workspaces: nothing is written behind the bytes that the query names, wherever the
matrices lie, and two captured graphs that share one are replayed in turns with eager calls between."""
import pytest

from operator_util import put
from paper_2310_14997_amd import binding as bd
from test_gpu_dense import ACTS, TYPES, d_of, inputs, t_of
from test_gpu_distill import dtype
from test_gpu_distill import inputs as rows_of_scores

pytestmark = pytest.mark.gpu
BEHIND = 1 << 16


def room(n):
    """n bytes of workspace, and a check of what lies behind them"""
    import torch
    buf = torch.full((n + BEHIND,), 0xA5, dtype=torch.uint8, device="cuda:0")

    def check():
        assert bool((buf[n:] == 0xA5).all()), "written behind the workspace"
    return (buf[:n] if n else None), check


def layer(R, I, O, types, act, shift=0):
    """(forward, backward, outputs, check) of a layer on one workspace"""
    import torch
    d = inputs(R, I, O, types, seed=4)
    ti, to = d_of(types[0]), d_of(types[1])
    cfg = bd.make_dense_config(R, I, O, t_of(types[0]), t_of(types[1]), ACTS[act])
    x, W, b, gy = put(d["x"], ti, shift), put(d["W"], ti, shift), put(d["bias"], ti, shift), put(d["grad_y"], to, shift)
    e = lambda t, *s: torch.empty(*s, dtype=t, device="cuda:0")
    y, z, gx, gW, gb = e(to, R, O), e(to, R, O), e(ti, R, I), e(ti, O, I), e(ti, O)
    ws, check = room(bd.spcfg_dense_workspace_bytes(cfg))
    return (lambda: bd.spcfg_dense_forward(cfg, x, W, b, None, y, z, ws),
            lambda: bd.spcfg_dense_backward(cfg, x, W, z, gy, None, gx, gW, gb, ws), (y, z, gx, gW, gb), check, x)


@pytest.mark.parametrize("types", TYPES, ids="-".join)
@pytest.mark.parametrize("R,I,O", [(2048, 512, 520), (1025, 263, 1111), (130, 2050, 700), (4100, 72, 130), (900, 2056, 2304),
                                   (70000, 24, 40)])
def test_layers_stay_inside(R, I, O, types):
    import torch
    for act in ("relu", "silu"):
        for shift in (0, 1):
            print("case workspace", R, I, O, types, act, shift, flush=True)
            forward, backward, _, check, _ = layer(R, I, O, types, act, shift)
            forward()
            backward()
            torch.cuda.synchronize()
            check()


@pytest.mark.parametrize("bf16", [False, True], ids=["fp32", "bf16"])
@pytest.mark.parametrize("R,V", [(1, 131071), (20, 70001), (70, 33000)])
def test_distillation_stays_inside(R, V, bf16):
    import torch
    s, t, ids, _ = rows_of_scores(R, V, 9, bf16)
    ws, check = room(bd.spcfg_distill_workspace_bytes(R, V))
    o = [torch.empty(R, device="cuda:0") for _ in range(2)]
    for shift in (0, 1):
        ts, tt, ti = put(s, dtype(bf16), shift), put(t, dtype(bf16), shift), put(ids, torch.int32, shift)
        bd.spcfg_distill_forward(ts, tt, ti, 1.0, *o, ws)
        bd.spcfg_distill_forward_backward(ts, tt, ti, 1.0, None, *o, torch.empty_like(ts), ws)
        torch.cuda.synchronize()
        check()


@pytest.mark.parametrize("types", TYPES[1:], ids="-".join)
def test_graphs_of_bf16_layers(types):
    """Off 16 bytes, so that planes of x, W and dz are all made; split sums; three replays on new inputs against eager calls."""
    import torch
    forward, backward, outs, check, x = layer(4100, 264, 328, types, "silu", 1)
    forward()
    backward()
    torch.cuda.synchronize()
    graphs = []
    for step in (forward, backward):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
        graphs.append(g)
    for turn in range(3):
        x.mul_(0.75)
        for t in outs:
            t.fill_(float("nan"))
        graphs[0].replay()
        graphs[1].replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        assert all(bool(torch.isfinite(t).all()) for t in got)
        forward()
        backward()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, got)), turn
    check()
