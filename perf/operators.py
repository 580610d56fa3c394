"""The library's operators around the grammar: the layers of the networks that make the rule scores, and losses with
their gradients - distillation of rows of scores from a teacher's top entries, and preferences between sentences by
their log Z.  Cases that can be timed, each operator in plain torch form, and (where `own` is true) as the library's call.

A case is a plain dict; `op` says which operator, the other keys are its sizes:
  "dense_forward"   y = act(x W^T + bias) + residual            rows, n_in, n_out, types, activation, bias, residual, keep
  "dense_backward"  gradients of x, W and bias from grad_y      the same; residual: grad_y is added to the gradient of x
  "distill"         loss and gradient of rows of scores         rows, V, k, type, temperature, ragged
  "distill_eval"    the loss alone
  "preference"      loss, margin and gradient in log Z          B sentences, pairs, beta, smoothing, reference
"""
from __future__ import annotations

import math

import torch

own = False

_TORCH = {"fp32": torch.float32, "bf16": torch.bfloat16}
_DENSE = dict(rows=1, n_in=1, n_out=1, in_type="fp32", out_type="fp32", activation="none", bias=True, residual=False,
              keep=False)
_DISTILL = dict(rows=1, V=2, k=1, type="fp32", temperature=1.0, ragged=False)
_PREFERENCE = dict(B=2, pairs=1, beta=0.1, smoothing=0.0, reference=True)


def _case(op, **kw):
    base = _DENSE if op.startswith("dense") else _DISTILL if op.startswith("distill") else _PREFERENCE
    assert set(kw) <= set(base) | {"name"}
    return {"op": op, **base, **kw}


def listed():
    return [
        # one residual layer over the nonterminals' embeddings of a tiny grammar: a launch and little else
        _case("dense_forward", name="layer_tiny", rows=30, n_in=512, n_out=512, activation="relu", residual=True),
        # emission scores of the headline grammar, in fp32, as the rule softmaxes take them
        _case("dense_forward", name="scores_fp32", rows=2048, n_in=512, n_out=10000, bias=False),
        # one residual layer over all symbols of the large grammar, bf16, with what its backward pass needs
        _case("dense_forward", name="layer_bf16", rows=8192, n_in=512, n_out=512, in_type="bf16", out_type="bf16",
              activation="relu", residual=True, keep=True),
        # a wide layer, where the matrix product is everything
        _case("dense_forward", name="wide_bf16", rows=8192, n_in=4096, n_out=4096, in_type="bf16", out_type="bf16",
              activation="gelu"),
        # gradients of a small layer whose sizes are multiples of nothing
        _case("dense_backward", name="layer_odd_back", rows=333, n_in=141, n_out=474, activation="silu"),
        # gradients of the residual layer over all symbols of the headline grammar, in fp32
        _case("dense_backward", name="layer_fp32_back", rows=4096, n_in=512, n_out=512, activation="relu", residual=True),
        # gradients of the emission scores: bf16 network, fp32 gradients from the rule softmaxes
        _case("dense_backward", name="scores_bf16_back", rows=2048, n_in=512, n_out=10000, in_type="bf16"),
        # a tiny grammar's emission rows learning from a teacher's best words
        _case("distill", name="distill_tiny", rows=60, V=200, k=8, temperature=2.0),
        # the headline grammar's emission table from a larger grammar's, rows with different numbers of kept words
        _case("distill", name="distill_words", rows=2048, V=10000, k=64, temperature=2.0, ragged=True),
        # a few rows over a long vocabulary, in bf16
        _case("distill", name="distill_long", rows=8, V=131071, k=128, type="bf16"),
        # a batch of sentences, each with one corrupted copy
        _case("preference", name="pairs_small", B=64, pairs=32),
        # a full batch, every sentence against several others
        _case("preference", name="pairs_many", B=960, pairs=8192, smoothing=0.1),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    """One more case: sizes, types and options of the listed ones' ranges, at no more than the largest one's cost."""
    ranks = [work(c) for c in listed()]
    most_flops, most_bytes = max(w["flops"] for w in ranks), max(w["bytes"] for w in ranks)
    while True:
        op = rng.choice(["dense_forward"] * 3 + ["dense_backward"] * 3 + ["distill"] * 2 + ["distill_eval", "preference"])
        if op.startswith("dense"):
            types = rng.choice([("fp32", "fp32"), ("bf16", "bf16"), ("bf16", "fp32")])
            n_in = _log_int(rng, 16, 4096)
            square = rng.random() < 0.4
            c = _case(op, rows=_log_int(rng, 1, 8192), n_in=n_in, n_out=n_in if square else _log_int(rng, 16, 10000),
                      in_type=types[0], out_type=types[1], bias=rng.random() < 0.7,
                      activation=rng.choice(["none", "relu", "gelu", "silu"]))
            c["residual"] = square and types[0] == types[1] and rng.random() < 0.6
            c["keep"] = op == "dense_forward" and c["activation"] != "none" and rng.random() < 0.5
        elif op.startswith("distill"):
            V = _log_int(rng, 30, 131072)
            c = _case(op, rows=_log_int(rng, 1, 8192), V=V, k=_log_int(rng, 1, min(V, 256)),
                      type=rng.choice(["fp32", "bf16"]), temperature=rng.choice([1.0, 2.0, 4.0]),
                      ragged=rng.random() < 0.5)
        else:
            c = _case(op, B=_log_int(rng, 2, 960), pairs=_log_int(rng, 1, 8192), beta=rng.choice([0.05, 0.1, 0.5]),
                      smoothing=rng.choice([0.0, 0.1]), reference=rng.random() < 0.7)
        w = work(c)
        if w["flops"] <= most_flops and w["bytes"] <= most_bytes:
            return c


def work(case):
    c = case
    size = {"fp32": 4, "bf16": 2}
    if c["op"].startswith("dense"):
        R, I, O = c["rows"], c["n_in"], c["n_out"]
        si, so = size[c["in_type"]], size[c["out_type"]]
        if c["op"] == "dense_forward":
            # x, W (bias, residual unless it is x) in; y (and the activation's input) out
            nbytes = si * (R * I + O * I + (O if c["bias"] else 0)) + so * R * O * (2 if c["keep"] else 1)
            return dict(bytes=nbytes, flops=2 * R * I * O)
        # x, W, grad_y (the activation's input) in; three gradients out
        nbytes = si * 2 * (R * I + O * I) + so * R * O * (1 if c["activation"] == "none" else 2)
        return dict(bytes=nbytes + (si * O if c["bias"] else 0), flops=4 * R * I * O)
    if c["op"].startswith("distill"):
        R, V, k, s = c["rows"], c["V"], c["k"], size[c["type"]]
        nbytes = s * R * V * (2 if c["op"] == "distill" else 1) + R * k * (s + 4) + 8 * R
        return dict(bytes=nbytes, flops=R * V * (6 if c["op"] == "distill" else 4))
    B, n = c["B"], c["pairs"]
    return dict(bytes=4 * (B * (3 if c["reference"] else 2) + 4 * n), flops=20 * n + 2 * B)


def prepare(case, seed):
    """Inputs on the GPU, made from the seed alone, and the buffers that a user's program keeps between calls."""
    dev = torch.device("cuda:0")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    c = case
    randn = lambda *shape: torch.randn(*shape, generator=gen, device=dev)
    empty = lambda dtype, *shape: torch.empty(*shape, dtype=dtype, device=dev)
    if c["op"].startswith("dense"):
        R, I, O = c["rows"], c["n_in"], c["n_out"]
        ti, to = _TORCH[c["in_type"]], _TORCH[c["out_type"]]
        st = dict(case=c, x=randn(R, I).to(ti), W=(randn(O, I) * math.sqrt(2.0 / (I + O))).to(ti),
                  bias=(0.1 * randn(O)).to(ti) if c["bias"] else None)
        if c["op"] == "dense_forward":
            st["residual"] = st["x"] if c["residual"] else None  # y = act(f(x)) + x
            st["y"], st["preact"] = empty(to, R, O), empty(to, R, O) if c["keep"] else None
            return st
        st["preact"] = None
        if c["activation"] != "none":  # as the forward pass kept it: an input here, whose signs relu's slope goes by
            z = st["x"].float() @ st["W"].float().t()
            st["preact"] = (z + st["bias"].float() if c["bias"] else z).to(to)
        st["grad_y"] = (0.01 * randn(R, O)).to(to)
        st["grads"] = [empty(ti, R, I), empty(ti, O, I), empty(ti, O) if c["bias"] else None]
        return st
    if c["op"].startswith("distill"):
        R, V, k, t = c["rows"], c["V"], c["k"], _TORCH[c["type"]]
        logits = 2.0 * randn(R, V)
        # a teacher that agrees with the student in part; its k best entries, best first
        best, ids = torch.topk(0.7 * logits + 1.4 * randn(R, V), k, dim=1)
        ids = ids.to(torch.int32)
        if c["ragged"]:  # rows keep between none and all of them; the others are marked absent
            kept = torch.randint(0, k + 1, (R, 1), generator=gen, device=dev)
            ids = torch.where(torch.arange(k, device=dev)[None, :] < kept, ids, -1)
        st = dict(case=c, logits=logits.to(t), teacher=best.to(t).contiguous(), ids=ids.contiguous(),
                  loss=empty(torch.float32, R), lse=empty(torch.float32, R))
        if c["op"] == "distill":
            st["grad_loss"] = torch.rand(R, generator=gen, device=dev) / R
            st["grad_logits"] = empty(t, R, V)
        return st
    B, n = c["B"], c["pairs"]
    words = torch.randint(2, 41, (B,), generator=gen, device=dev).float()
    st = dict(case=c, logZ=-6.0 * words + 4.0 * randn(B))
    st["ref"] = st["logZ"] + 3.0 * randn(B) if c["reference"] else None
    st["chosen"] = torch.randint(0, B, (n,), generator=gen, device=dev, dtype=torch.int32)
    other = torch.randint(1, B, (n,), generator=gen, device=dev, dtype=torch.int32)
    st["rejected"] = ((st["chosen"] + other) % B).to(torch.int32).contiguous()
    st["grad_loss"] = torch.full((n,), 1.0 / n, device=dev)
    st["loss"], st["margin"] = empty(torch.float32, n), empty(torch.float32, n)
    st["grad_logZ"] = empty(torch.float32, B)
    return st


def run(state):
    """One pass: the operator's outputs."""
    op = state["case"]["op"]
    if own:
        return _OWN[op](state)
    return _PLAIN[op](state)


# ---- plain forms: elementary operations in 32 bits, rounded once at the end ---------------------------------------

_SQRT_HALF = math.sqrt(0.5)


def _act(z, kind):
    if kind == "relu":
        return torch.clamp(z, min=0.0)
    if kind == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * _SQRT_HALF))
    if kind == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _act_slope(z, kind):
    if kind == "relu":
        return (z > 0.0).to(z.dtype)
    if kind == "gelu":
        return 0.5 * (1.0 + torch.erf(z * _SQRT_HALF)) + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    if kind == "silu":
        s = 1.0 / (1.0 + torch.exp(-z))
        return s * (1.0 + z * (1.0 - s))
    return torch.ones_like(z)


def _plain_dense_forward(s):
    c = s["case"]
    out = _TORCH[c["out_type"]]
    z = s["x"].float() @ s["W"].float().t()
    if s["bias"] is not None:
        z = z + s["bias"].float()
    y = _act(z, c["activation"])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    res = dict(y=y.to(out))
    if c["keep"]:
        res["preact"] = z.to(out)
    return res


def _plain_dense_backward(s):
    c = s["case"]
    t = _TORCH[c["in_type"]]
    gy = s["grad_y"].float()
    dz = gy if c["activation"] == "none" else gy * _act_slope(s["preact"].float(), c["activation"])
    gx = dz @ s["W"].float()
    if c["residual"]:
        gx = gx + gy
    res = dict(grad_x=gx.to(t), grad_W=(dz.t() @ s["x"].float()).to(t))
    if s["bias"] is not None:
        res["grad_bias"] = dz.sum(0).to(t)
    return res


def _plain_distill(s, gradient=True):
    c = s["case"]
    tau = c["temperature"]
    z = s["logits"].float() / tau
    top = z.max(dim=1, keepdim=True).values
    e = torch.exp(z - top)
    total = e.sum(dim=1, keepdim=True)
    lse = top + torch.log(total)
    there = s["ids"] >= 0
    ids = torch.where(there, s["ids"], 0).long()
    a = torch.where(there, s["teacher"].float() / tau, -math.inf)
    some = there.any(dim=1, keepdim=True)
    a_top = torch.where(some, a.max(dim=1, keepdim=True).values, 0.0)
    w = torch.exp(a - a_top)
    w_total = torch.where(some, w.sum(dim=1, keepdim=True), 1.0)
    p = w / w_total
    log_p = a - a_top - torch.log(w_total)
    log_q = torch.gather(z, 1, ids) - lse
    loss = tau * tau * torch.where(there, p * (log_p - log_q), 0.0).sum(dim=1)
    res = dict(loss=loss, lse=lse[:, 0])
    if gradient:
        g = torch.where(some, s["grad_loss"][:, None] * tau, 0.0)
        d = (e / total) * g
        d.scatter_add_(1, ids, -g * p)
        res["grad_logits"] = d.to(_TORCH[c["type"]])
    return res


def _plain_preference(s):
    c = s["case"]
    beta, eps = c["beta"], c["smoothing"]
    ratio = s["logZ"].double()
    if s["ref"] is not None:
        ratio = ratio - s["ref"].double()
    i, j = s["chosen"].long(), s["rejected"].long()
    margin = (ratio[i] - ratio[j]).float()
    x = beta * margin
    tail = torch.log1p(torch.exp(-x.abs()))
    loss = (1.0 - eps) * (torch.clamp(-x, min=0.0) + tail) + eps * (torch.clamp(x, min=0.0) + tail)
    up = 1.0 / (1.0 + torch.exp(-x))
    down = 1.0 / (1.0 + torch.exp(x))
    w = (beta * (eps * up - (1.0 - eps) * down) * s["grad_loss"]).double()
    grad = torch.zeros(c["B"], dtype=torch.float64, device=w.device)
    grad.index_add_(0, i, w).index_add_(0, j, -w)
    return dict(loss=loss, margin=margin, grad_logZ=grad.float())


_PLAIN = {"dense_forward": _plain_dense_forward, "dense_backward": _plain_dense_backward, "distill": _plain_distill,
          "distill_eval": lambda s: _plain_distill(s, gradient=False), "preference": _plain_preference}


# ---- the library's calls -------------------------------------------------------------------------------------------

def _dense_config(s, bd):
    """Configuration and workspace of a layer: made once, kept beside its weights."""
    if "config" not in s:
        c = s["case"]
        types = {"fp32": bd.TYPE_F32, "bf16": bd.TYPE_BF16}
        acts = {"none": bd.ACT_NONE, "relu": bd.ACT_RELU, "gelu": bd.ACT_GELU, "silu": bd.ACT_SILU}
        s["config"] = bd.make_dense_config(c["rows"], c["n_in"], c["n_out"], types[c["in_type"]], types[c["out_type"]],
                                           acts[c["activation"]])
        s["workspace"] = torch.empty(bd.spcfg_dense_workspace_bytes(s["config"]), dtype=torch.uint8, device=s["x"].device)
    return s["config"], s["workspace"]


def _own_dense_forward(s):
    from paper_2310_14997_amd import binding as bd
    cfg, ws = _dense_config(s, bd)
    bd.spcfg_dense_forward(cfg, s["x"], s["W"], s["bias"], s["residual"], s["y"], s["preact"], ws)
    return dict(y=s["y"], preact=s["preact"]) if s["case"]["keep"] else dict(y=s["y"])


def _own_dense_backward(s):
    from paper_2310_14997_amd import binding as bd
    cfg, ws = _dense_config(s, bd)
    gx, gW, gb = s["grads"]
    bd.spcfg_dense_backward(cfg, s["x"], s["W"], s["preact"], s["grad_y"], s["grad_y"] if s["case"]["residual"] else None,
                            gx, gW, gb, ws)
    return dict(grad_x=gx, grad_W=gW) if gb is None else dict(grad_x=gx, grad_W=gW, grad_bias=gb)


def _distill_workspace(s, bd):
    if "workspace" not in s:
        c = s["case"]
        n = bd.spcfg_distill_workspace_bytes(c["rows"], c["V"])
        s["workspace"] = torch.empty(n, dtype=torch.uint8, device=s["logits"].device)
    return s["workspace"]


def _own_distill(s):
    from paper_2310_14997_amd import binding as bd
    bd.spcfg_distill_forward_backward(s["logits"], s["teacher"], s["ids"], s["case"]["temperature"], s["grad_loss"],
                                      s["loss"], s["lse"], s["grad_logits"], _distill_workspace(s, bd))
    return dict(loss=s["loss"], lse=s["lse"], grad_logits=s["grad_logits"])


def _own_distill_eval(s):
    from paper_2310_14997_amd import binding as bd
    bd.spcfg_distill_forward(s["logits"], s["teacher"], s["ids"], s["case"]["temperature"], s["loss"], s["lse"],
                             _distill_workspace(s, bd))
    return dict(loss=s["loss"], lse=s["lse"])


def _own_preference(s):
    from paper_2310_14997_amd import binding as bd
    c = s["case"]
    bd.spcfg_preference_forward_backward(s["logZ"], s["ref"], s["chosen"], s["rejected"], c["beta"], c["smoothing"],
                                         s["grad_loss"], s["loss"], s["margin"], s["grad_logZ"])
    return dict(loss=s["loss"], margin=s["margin"], grad_logZ=s["grad_logZ"])


_OWN = {"dense_forward": _own_dense_forward, "dense_backward": _own_dense_backward, "distill": _own_distill,
        "distill_eval": _own_distill_eval, "preference": _own_preference}


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------

def exact(case, seed):
    """What run() returns for these inputs, in 64 bits."""
    c, s = case, prepare(case, seed)
    d = lambda t: t.to(torch.float64)
    if c["op"].startswith("dense"):
        kind = c["activation"]
        if c["op"] == "dense_forward":
            z = torch.mm(d(s["x"]), d(s["W"]).t().contiguous())
            z = z if s["bias"] is None else z.add_(d(s["bias"]))
            y = (z if kind == "none" else z * (z > 0) if kind == "relu" else z * torch.sigmoid(z) if kind == "silu"
                 else z * torch.special.ndtr(z))
            y = y if s["residual"] is None else y + d(s["residual"])
            return dict(y=y, preact=z) if c["keep"] else dict(y=y)
        dz = d(s["grad_y"])
        if kind != "none":
            z = d(s["preact"])
            if kind == "relu":
                dz = torch.where(z > 0, dz, 0.0)
            elif kind == "silu":
                dz = dz * (torch.sigmoid(z) + z * torch.sigmoid(z) * torch.sigmoid(-z))
            else:
                dz = dz * (torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi))
        gx = torch.mm(dz, d(s["W"]))
        out = dict(grad_x=gx + d(s["grad_y"]) if c["residual"] else gx, grad_W=torch.mm(dz.t().contiguous(), d(s["x"])))
        if s["bias"] is not None:
            out["grad_bias"] = dz.sum(dim=0)
        return out
    if c["op"].startswith("distill"):
        tau = c["temperature"]
        log_q = torch.log_softmax(d(s["logits"]) / tau, dim=1)
        lse = torch.logsumexp(d(s["logits"]) / tau, dim=1)
        # the teacher's distribution over the whole row: zero outside its kept entries
        target = torch.zeros_like(log_q)
        mask = s["ids"] >= 0
        p = torch.nan_to_num(torch.softmax(torch.where(mask, d(s["teacher"]) / tau, -math.inf), dim=1))
        target.scatter_add_(1, s["ids"].long().clamp(min=0), p)
        loss = tau ** 2 * (torch.special.xlogy(p, p).sum(dim=1) - torch.where(target > 0, target * log_q, 0.0).sum(dim=1))
        out = dict(loss=loss, lse=lse)
        if c["op"] == "distill":
            g = d(s["grad_loss"])[:, None] * mask.any(dim=1)[:, None]
            out["grad_logits"] = g * tau * (torch.exp(log_q) - target)
        return out
    ratio = d(s["logZ"]) - (0.0 if s["ref"] is None else d(s["ref"]))
    pick = lambda idx: torch.nn.functional.one_hot(idx.long(), c["B"]).to(torch.float64)
    sign = pick(s["chosen"]) - pick(s["rejected"])  # [pairs, B]
    margin = sign @ ratio
    x = c["beta"] * margin
    loss = -(1 - c["smoothing"]) * torch.nn.functional.logsigmoid(x) - c["smoothing"] * torch.nn.functional.logsigmoid(-x)
    w = c["beta"] * (torch.sigmoid(x) - (1 - c["smoothing"])) * d(s["grad_loss"])
    return dict(loss=loss, margin=margin, grad_logZ=w @ sign)
