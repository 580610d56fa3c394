"""A whole training step of a neural grammar in the library's calls: embeddings through residual layers and score products,
the rule softmaxes, the inside pass, a preference loss on pairs of sentences plus distillation of the emission rows, and back
to the gradients of every weight - against the same step of the 64-bit oracles, and against differences of the loss."""
import numpy as np
import pytest

from oracle import losses_oracle as LO
from oracle import network_oracle as NO
from oracle import rules_oracle as RO
from oracle import spcfg_oracle as O
from operator_util import put, values
from paper_2310_14997_amd import binding as bd
from parity_util import check_grad

pytestmark = pytest.mark.gpu

D, N, P, V, B, N_MAX, K = 48, 40, 56, 120, 8, 9, 6
M = N + P
LENGTHS = np.array([9, 7, 5, 9, 4, 6, 3, 8], np.int32)
CHOSEN, REJECTED = np.array([0, 1, 2, 3, 0], np.int32), np.array([4, 5, 6, 7, 1], np.int32)
BETA, EPS, TAU, W_DISTILL = 0.2, 0.05, 2.0, 0.3


def model(rng):
    """Embeddings of nonterminals and preterminals, one residual layer each, and the tables that the scores are products with."""
    n = lambda *s: (rng.normal(size=s)).astype(np.float32)
    return dict(E_N=n(N, D), E_P=n(P, D), W_N=0.2 * n(D, D), b_N=0.1 * n(D), W_P=0.2 * n(D, D), b_P=0.1 * n(D),
                T_root=0.3 * n(1, D), T_L=0.3 * n(M, D), T_R=0.3 * n(M, D), T_V=0.3 * n(V, D))


def oracle_step(w, tokens, teacher, ids, ref):
    w = {k: np.asarray(v, np.float64) for k, v in w.items()}
    hN, zN = NO.forward(w["E_N"], w["W_N"], w["b_N"], w["E_N"], "relu")
    hP, zP = NO.forward(w["E_P"], w["W_P"], w["b_P"], w["E_P"], "relu")
    root = NO.forward(hN, w["T_root"])[0][:, 0]
    sL, sR, sV = (NO.forward(h, w[t])[0] for h, t in ((hN, "T_L"), (hN, "T_R"), (hP, "T_V")))
    f = RO.forward(root, sL, sR, sV, tokens, LENGTHS)
    gout = O.inside_backward(f["log_root"], f["L"], f["R"], f["log_emit"], LENGTHS)
    loss_p, _, gz = LO.preference(gout["logZ"], ref, CHOSEN, REJECTED, BETA, EPS)
    loss_d, _, gV = LO.distill(sV, teacher, ids, TAU, np.full(P, W_DISTILL))
    total = loss_p.sum() + W_DISTILL * loss_d.sum()
    g = O.inside_backward(f["log_root"], f["L"], f["R"], f["log_emit"], LENGTHS, gz)
    b = RO.backward(root, sL, sR, sV, tokens, LENGTHS, g["grad_log_root"], g["grad_L"], g["grad_R"], g["grad_log_emit"])
    out, ghN, ghP = {}, 0.0, 0.0
    for name, h, gs in (("T_root", "N", b["grad_root_logits"][:, None]), ("T_L", "N", b["grad_L_logits"]),
                        ("T_R", "N", b["grad_R_logits"]), ("T_V", "P", b["grad_emis_logits"] + gV)):
        gh, out[name], _ = NO.backward(hN if h == "N" else hP, w[name], None, gs)
        ghN, ghP = (ghN + gh, ghP) if h == "N" else (ghN, ghP + gh)
    out["E_N"], out["W_N"], out["b_N"] = NO.backward(w["E_N"], w["W_N"], zN, ghN, "relu", ghN)
    out["E_P"], out["W_P"], out["b_P"] = NO.backward(w["E_P"], w["W_P"], zP, ghP, "relu", ghP)
    return total, out


def library_step(w, tokens, teacher, ids, ref):
    import torch
    f = torch.float32
    t = {k: put(v, f) for k, v in w.items()}
    e = lambda *s: torch.empty(*s, device="cuda:0")
    tok, tt, ti, tref = put(tokens, torch.int32), put(teacher, f), put(ids, torch.int32), put(ref, f)
    layer = {s: bd.make_dense_config(n, D, D, activation=bd.ACT_RELU) for s, n in (("N", N), ("P", P))}
    score = {k: bd.make_dense_config(n, D, o) for k, n, o in (("T_root", N, 1), ("T_L", N, M), ("T_R", N, M), ("T_V", P, V))}
    need = max(bd.spcfg_dense_workspace_bytes(c) for c in list(layer.values()) + list(score.values()))
    ws = torch.empty(need, dtype=torch.uint8, device="cuda:0") if need else None
    h, z, s = {}, {}, {}
    for k, n in (("N", N), ("P", P)):
        h[k], z[k] = e(n, D), e(n, D)
        bd.spcfg_dense_forward(layer[k], t["E_" + k], t["W_" + k], t["b_" + k], t["E_" + k], h[k], z[k], ws)
    for k, c in score.items():
        s[k] = e(c.rows, c.n_out)
        bd.spcfg_dense_forward(c, h["P" if k == "T_V" else "N"], t[k], None, None, s[k], None, ws)
    log_root, L, R, log_emit, lse = e(N), e(N, M), e(N, M), e(B, N_MAX, P), e(P)
    bd.spcfg_rules_forward(s["T_root"].view(N), s["T_L"], s["T_R"], s["T_V"], tok, LENGTHS, log_root, L, R, log_emit, lse)
    cfg = bd.make_config(N, P, B, N_MAX)
    iws = torch.empty(bd.spcfg_workspace_bytes_for(cfg, LENGTHS, N_MAX), dtype=torch.uint8, device="cuda:0")
    logZ = e(B)
    bd.spcfg_inside(cfg, log_root, L, R, log_emit, LENGTHS, logZ, iws)
    n = len(CHOSEN)
    lp, mp, gz = e(n), e(n), e(B)
    bd.spcfg_preference_forward_backward(logZ, tref, put(CHOSEN, torch.int32), put(REJECTED, torch.int32), BETA, EPS, None, lp,
                                         mp, gz)
    gL, gR, gr, ge = e(N, M), e(N, M), e(N), e(B, N_MAX, P)
    bd.spcfg_inside_backward(cfg, log_root, L, R, log_emit, LENGTHS, gz, gL, gR, gr, ge, iws)
    gs = {"T_root": e(N, 1), "T_L": e(N, M), "T_R": e(N, M), "T_V": e(P, V)}
    bd.spcfg_rules_backward(log_root, L, R, s["T_V"], lse, tok, LENGTHS, gr, gL, gR, ge, gs["T_root"].view(N), gs["T_L"],
                            gs["T_R"], gs["T_V"], e(32, P))
    ld, le, gd = e(P), e(P), e(P, V)
    bd.spcfg_distill_forward_backward(s["T_V"], tt, ti, TAU, torch.full((P,), W_DISTILL, device="cuda:0"), ld, le, gd, None)
    gs["T_V"] += gd
    out, gh = {}, {}
    for k, c in score.items():
        side = "P" if k == "T_V" else "N"
        out[k] = e(c.n_out, D)
        g = e(c.rows, D)
        bd.spcfg_dense_backward(c, h[side], t[k], None, gs[k], gh.get(side), g, out[k], None, ws)
        gh[side] = g
    for k, n in (("N", N), ("P", P)):
        out["E_" + k], out["W_" + k], out["b_" + k] = e(n, D), e(D, D), e(D)
        bd.spcfg_dense_backward(layer[k], t["E_" + k], t["W_" + k], z[k], gh[k], gh[k], out["E_" + k], out["W_" + k],
                                out["b_" + k], ws)
    total = lp.double().sum() + W_DISTILL * ld.double().sum()
    return float(total), {k: values(v) for k, v in out.items()}


def data(seed):
    rng = np.random.default_rng(seed)
    w = model(rng)
    tokens = np.full((B, N_MAX), -1, np.int32)
    for b in range(B):
        tokens[b, :LENGTHS[b]] = rng.integers(0, V, size=LENGTHS[b])
    teacher = rng.normal(size=(P, K)).astype(np.float32)
    ids = np.stack([rng.choice(V, size=K, replace=False) for _ in range(P)]).astype(np.int32)
    ids[3, 2:] = -1
    return w, tokens, teacher, ids, (-40 + 3 * rng.normal(size=B)).astype(np.float32)


def test_against_the_oracles():
    w, tokens, teacher, ids, ref = data(11)
    want_total, want = oracle_step(w, tokens, teacher, ids, ref)
    total, got = library_step(w, tokens, teacher, ids, ref)
    assert abs(total - want_total) <= 2e-5 * abs(want_total)
    assert set(got) == set(want)
    for k in sorted(want):  # the inside pass's own gradient tolerance, twice (it and the layers below it)
        check_grad(k, got[k], want[k].reshape(got[k].shape), 2e-4)


def test_against_differences():
    """The oracle's step is itself the gradient of its loss: differences along random directions, all weights at once."""
    w, tokens, teacher, ids, ref = data(12)
    w = {k: v.astype(np.float64) for k, v in w.items()}
    _, got = library_step(w, tokens, teacher, ids, ref)
    rng = np.random.default_rng(1)
    for _ in range(3):
        d = {k: rng.normal(size=v.shape) for k, v in w.items()}
        h = 1e-6
        up, _ = oracle_step({k: w[k] + h * d[k] for k in w}, tokens, teacher, ids, ref)
        down, _ = oracle_step({k: w[k] - h * d[k] for k in w}, tokens, teacher, ids, ref)
        along = sum(float((got[k].reshape(d[k].shape) * d[k]).sum()) for k in w)
        size = np.sqrt(sum(float((got[k] ** 2).sum()) for k in w))
        assert abs((up - down) / (2 * h) - along) <= 2e-4 * size + 1e-5
