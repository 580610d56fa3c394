"""CPU oracle for the losses around the grammar.  TEST INFRASTRUCTURE ONLY.

Distillation, row by row: p = softmax(teacher / tau) over the entries that are there (id >= 0, score above -inf),
q = softmax(logits / tau): loss = tau^2 sum_e p_e (log p_e - log q_id(e)), gradient tau (q - p at its ids); a row
without entries is 0 and 0, and one of nothing but -inf has lse -inf and, with entries, NaN.

Preference: margin = (logZ_c - ref_c) - (logZ_r - ref_r), x = beta margin, loss = (1 - eps) log(1 + exp(-x)) +
eps log(1 + exp(x)), gradient in logZ; absent pairs (a negative index) are 0.

Double precision, numpy; shares no code with the HIP path.  Pinned in tests/test_losses_oracle.py (finite differences,
hand-worked values).
"""
from __future__ import annotations

import numpy as np


def distill(logits, teacher, ids, tau, grad_loss=None):
    """(loss [rows], lse [rows], grad_logits [rows, V])"""
    s = np.asarray(logits, np.float64) / tau
    R, V = s.shape
    loss, lse, grad = np.zeros(R), np.zeros(R), np.zeros((R, V))
    for r in range(R):
        m = s[r].max()
        if m == -np.inf:  # nothing that the row could be
            lse[r], loss[r], grad[r] = m, np.nan, np.nan
            if not any(ids[r][e] >= 0 and teacher[r][e] > -np.inf for e in range(len(ids[r]))):
                loss[r], grad[r] = 0.0, 0.0
            continue
        lse[r] = m + np.log(np.exp(s[r] - m).sum())
        there = [e for e in range(len(ids[r])) if ids[r][e] >= 0 and teacher[r][e] > -np.inf]
        if not there:
            continue
        a = np.array([float(teacher[r][e]) for e in there]) / tau
        log_p = a - (a.max() + np.log(np.exp(a - a.max()).sum()))
        p = np.exp(log_p)
        at = np.array([ids[r][e] for e in there])
        live = p > 0
        loss[r] = tau ** 2 * (p[live] * (log_p[live] - (s[r][at[live]] - lse[r]))).sum()
        g = tau * np.exp(s[r] - lse[r])
        np.subtract.at(g, at, tau * p)
        grad[r] = g * (1.0 if grad_loss is None else float(grad_loss[r]))
    return loss, lse, grad


def preference(logZ, ref, chosen, rejected, beta, eps, grad_loss=None):
    """(loss [pairs], margin [pairs], grad_logZ [B])"""
    z = np.asarray(logZ, np.float64) - (0.0 if ref is None else np.asarray(ref, np.float64))
    n = len(chosen)
    loss, margin, grad = np.zeros(n), np.zeros(n), np.zeros(len(z))
    for p in range(n):
        c, r = chosen[p], rejected[p]
        if c < 0 or r < 0:
            continue
        margin[p] = z[c] - z[r]
        x = beta * margin[p]
        loss[p] = (1 - eps) * np.logaddexp(0.0, -x) + eps * np.logaddexp(0.0, x)
        up = np.exp(-np.logaddexp(0.0, -x))
        w = beta * (up - (1 - eps)) * (1.0 if grad_loss is None else float(grad_loss[p]))
        grad[c] += w
        grad[r] -= w
    return loss, margin, grad
