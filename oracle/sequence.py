"""float64 reference of the sequence and answer operators: the gated leaky
integrator with its gradient and single step, and the token log probabilities
and the distillation loss with their gradients, written from the formulas one
step and one row at a time (numpy, no code shared with the library)."""
from __future__ import annotations

import numpy as np

TAIL_MIN = 2.0 ** -20


def _gate(f):
    """(sigmoid(f), 1 - sigmoid(f)) without cancellation or overflow."""
    e = np.exp(-np.abs(f))
    a, b = 1.0 / (1.0 + e), e / (1.0 + e)
    return np.where(f >= 0, a, b), np.where(f >= 0, b, a)


def _steps(length, B, T):
    return np.full(B, T) if length is None else np.clip(np.asarray(length, np.int64), 0, T)


def gated_scan(x, f, length=None, h_first=None, coupled=True):
    """Returns h [B, T, D] (0 past a sample's length), h_last [B, D] and the
    state entering every step [B, T, D] (frozen past the length)."""
    x, f = np.asarray(x, np.float64), np.asarray(f, np.float64)
    B, T, D = x.shape
    n = _steps(length, B, T)
    state = np.zeros((B, D)) if h_first is None else np.array(h_first, np.float64)
    h, before = np.zeros((B, T, D)), np.zeros((B, T, D))
    for b in range(B):
        for t in range(T):
            before[b, t] = state[b]
            if t < n[b]:
                a, na = _gate(f[b, t])
                state[b] = a * state[b] + (na * x[b, t] if coupled else x[b, t])
                h[b, t] = state[b]
    return h, state, before


def gated_scan_grad(x, f, grad_h=None, grad_last=None, length=None, h_first=None, coupled=True):
    """Returns grad_x, grad_f [B, T, D] and grad_h_first [B, D] of
    sum(grad_h h) + sum(grad_last h_last)."""
    x, f = np.asarray(x, np.float64), np.asarray(f, np.float64)
    B, T, D = x.shape
    n = _steps(length, B, T)
    _, _, before = gated_scan(x, f, length, h_first, coupled)
    gx, gf = np.zeros((B, T, D)), np.zeros((B, T, D))
    lam = np.zeros((B, D)) if grad_last is None else np.array(grad_last, np.float64)
    for b in range(B):
        for t in range(n[b] - 1, -1, -1):
            if grad_h is not None:
                lam[b] += np.asarray(grad_h[b, t], np.float64)
            a, na = _gate(f[b, t])
            gx[b, t] = lam[b] * na if coupled else lam[b]
            gf[b, t] = lam[b] * a * na * (before[b, t] - x[b, t] if coupled else before[b, t])
            lam[b] = lam[b] * a
    return gx, gf, lam


def gated_step(x, f, state, slot=None, coupled=True):
    """Returns h [B, D] and the states after the step."""
    x, f, state = np.asarray(x, np.float64), np.asarray(f, np.float64), np.array(state, np.float64)
    h = np.zeros_like(x)
    for b in range(x.shape[0]):
        s = b if slot is None else int(slot[b])
        if 0 <= s < state.shape[0]:
            a, na = _gate(f[b])
            state[s] = a * state[s] + (na * x[b] if coupled else x[b])
            h[b] = state[s]
    return h, state


def _row(z):
    """(log probabilities, lse, whether the row has any mass) of one row."""
    if np.isnan(z).any() or np.isposinf(z).any():
        return np.full_like(z, np.nan), np.nan, True
    m = z.max()
    if np.isneginf(m):
        return np.full_like(z, -np.inf), -np.inf, False
    ls = np.log(np.exp(z - m).sum())
    return (z - m) - ls, m + ls, True          # m + ls alone would lose ls next to a huge m


def _plogp(p, logp):
    return np.where(p > 0, p * np.where(p > 0, logp, 0.0), np.where(np.isnan(p), p, 0.0))


def token_logprobs(logits, tokens=None, k=0, temperature=1.0, grad_logp=None, grad_entropy=None):
    """Returns a dict of logp, entropy, lse [R], top_logp, top_idx [R, k] and
    grad [R, V]."""
    x = np.asarray(logits, np.float64)
    R, V = x.shape
    out = {"logp": np.zeros(R), "entropy": np.zeros(R), "lse": np.zeros(R), "top_logp": np.zeros((R, k)),
           "top_idx": np.zeros((R, k), np.int64), "grad": np.zeros((R, V))}
    for r in range(R):
        logp, lse, mass = _row(x[r] / temperature)
        p = np.exp(logp)
        H = -_plogp(p, logp).sum()
        out["entropy"][r], out["lse"][r] = H, lse
        # largest first, ties by index, NaN below -infinity
        rank = np.where(np.isnan(x[r]), -np.inf, x[r])
        order = np.lexsort((np.arange(V), np.isnan(x[r]), -rank))[:k]
        out["top_idx"][r], out["top_logp"][r] = order, logp[order]
        tok = -1 if tokens is None else int(tokens[r])
        there = 0 <= tok < V
        if there:
            out["logp"][r] = logp[tok]
        g = float(grad_logp[r]) if there and grad_logp is not None else 0.0
        e = float(grad_entropy[r]) if grad_entropy is not None else 0.0
        if mass:
            v = -g * p - e * (_plogp(p, logp) + p * H)
            if there:
                v[tok] += g
            out["grad"][r] = v / temperature
    return out


def distill_top(logits, teacher_logp, teacher_idx, temperature=1.0, tail=False, weight=None):
    """Returns loss [R] and grad [R, V] of sum_r weight_r loss_r."""
    x = np.asarray(logits, np.float64)
    R, V = x.shape
    loss, grad = np.zeros(R), np.zeros((R, V))
    for r in range(R):
        use = [i for i in range(teacher_idx.shape[1]) if 0 <= int(teacher_idx[r, i]) < V]
        j = np.array([int(teacher_idx[r, i]) for i in use], np.int64)
        lq = np.array([float(teacher_logp[r, i]) for i in use], np.float64)
        if not (lq > -np.inf).any() and not np.isnan(lq).any():
            continue
        if not tail:                                # relative to the largest: unlikely classes have a mass too
            lq = lq - np.fmax.reduce(lq)
            lq = lq - np.log(np.exp(lq).sum())
        q = np.exp(lq)
        total = q.sum()
        logp, _, mass = _row(x[r] / temperature)
        p = np.exp(logp)
        listed = np.zeros(V, bool)
        listed[j] = True
        with np.errstate(divide="ignore", invalid="ignore"):
            loss[r] = sum(qi * (li - logp[ji]) for qi, li, ji in zip(q, lq, j) if qi > 0 or np.isnan(qi))
        q_rest, share = 0.0, None
        if tail and 1.0 - total >= TAIL_MIN and not listed.all():
            q_rest = 1.0 - total
            # by their own largest logit: next to the row's they may all be 0
            within, log_rest, some = _row(logp[~listed])
            loss[r] += q_rest * (np.log(q_rest) - log_rest)
            share = np.exp(within) if some else None
        if mass:
            v = p * ((total if tail else 1.0) + q_rest)
            np.subtract.at(v, j, q)
            if share is not None:
                v[~listed] -= q_rest * share
            grad[r] = v * ((1.0 if weight is None else float(weight[r])) / temperature)
    return loss, grad
