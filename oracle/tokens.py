"""float64 reference of the operators of models over tokens: rows of a table
by token, the short causal convolution and the selective state space scan, each
with its gradient, written from the formulas one step at a time (numpy, no code
shared with the library)."""
from __future__ import annotations

import numpy as np


def steps(length, B, T):
    return np.full(B, T) if length is None else np.clip(np.asarray(length, np.int64), 0, T)


def _places(tokens, V, length):
    """The places (b, t) that name a row."""
    B, T = tokens.shape
    n = steps(length, B, T)
    return [(b, t) for b in range(B) for t in range(n[b]) if 0 <= tokens[b, t] < V]


def embed(tokens, W, scale=1.0, length=None):
    out = np.zeros((*tokens.shape, W.shape[1]))
    for b, t in _places(tokens, W.shape[0], length):
        out[b, t] = scale * W[tokens[b, t]]
    return out


def embed_grad(tokens, grad, V, scale=1.0, length=None):
    """Returns the table's gradient and the sum of magnitudes behind each of
    its elements."""
    g, mag = np.zeros((V, grad.shape[2])), np.zeros((V, grad.shape[2]))
    for b, t in _places(tokens, V, length):
        g[tokens[b, t]] += scale * grad[b, t]
        mag[tokens[b, t]] += np.abs(scale * grad[b, t])
    return g, mag


def sigmoid(v):
    e = np.exp(-np.abs(v))
    return np.where(v >= 0, 1.0, e) / (1.0 + e)


def softplus(v):
    return np.maximum(v, 0) + np.log1p(np.exp(-np.abs(v)))


def causal_conv(x, w, bias=None, length=None, x_first=None, silu=True):
    """Returns y [B, T, D] and the last K - 1 inputs [B, K - 1, D]."""
    B, T, D = x.shape
    K = w.shape[1]
    y, last = np.zeros((B, T, D)), np.zeros((B, K - 1, D))
    for b, n in enumerate(steps(length, B, T)):
        seen = np.concatenate([np.zeros((K - 1, D)) if x_first is None else x_first[b], x[b, :n]])
        for t in range(n):
            c = (w.T * seen[t:t + K]).sum(0) + (0 if bias is None else bias)
            y[b, t] = c * sigmoid(c) if silu else c
        last[b] = seen[n:]
    return y, last


def causal_conv_grad(x, w, grad_y, bias=None, length=None, x_first=None, grad_last=None, silu=True):
    """Returns the gradients of x, w, bias and x_first."""
    B, T, D = x.shape
    K = w.shape[1]
    gx, g0, gw, gb = np.zeros((B, T, D)), np.zeros((B, K - 1, D)), np.zeros((D, K)), np.zeros(D)
    for b, n in enumerate(steps(length, B, T)):
        seen = np.concatenate([np.zeros((K - 1, D)) if x_first is None else x_first[b], x[b, :n]])
        gs = np.zeros_like(seen)
        if grad_last is not None:
            gs[n:] += grad_last[b]
        for t in range(n):
            c = (w.T * seen[t:t + K]).sum(0) + (0 if bias is None else bias)
            s = sigmoid(c)
            gc = grad_y[b, t] * (s * (1 + c * (1 - s)) if silu else 1.0)
            gs[t:t + K] += w.T * gc
            gw += (seen[t:t + K] * gc).T
            gb += gc
        gx[b, :n], g0[b] = gs[K - 1:], gs[:K - 1]
    return gx, gw, gb, g0


def selective_scan(x, dt, A, B, C, D=None, z=None, dt_bias=None, length=None, h_first=None, softplus_=True):
    """B and C are [B, T, G, N].  Returns y [B, T, D], h_last [B, D, N] and the
    state before every step [B, T, D, N]."""
    nb, T, W = x.shape
    G, N = B.shape[2:]
    of = np.arange(W) // (W // G)
    y, before = np.zeros((nb, T, W)), np.zeros((nb, T, W, N))
    last = np.zeros((nb, W, N)) if h_first is None else np.array(h_first, np.float64)
    for b, n in enumerate(steps(length, nb, T)):
        h = last[b]
        for t in range(T):
            before[b, t] = h
            if t >= n:
                continue
            r = dt[b, t] + (0 if dt_bias is None else dt_bias)
            delta = softplus(r) if softplus_ else r
            h = np.exp(delta[:, None] * A) * h + (delta * x[b, t])[:, None] * B[b, t][of]
            v = (C[b, t][of] * h).sum(1) + (0 if D is None else D * x[b, t])
            y[b, t] = v if z is None else v * z[b, t] * sigmoid(z[b, t])
        last[b] = h
    return y, last, before


def selective_scan_grad(x, dt, A, B, C, grad_y, D=None, z=None, dt_bias=None, length=None, h_first=None,
                        grad_last=None, softplus_=True):
    """Returns a dict of the gradients of every input."""
    nb, T, W = x.shape
    G, N = B.shape[2:]
    of = np.arange(W) // (W // G)
    _, _, before = selective_scan(x, dt, A, B, C, D, z, dt_bias, length, h_first, softplus_)
    g = {"x": np.zeros((nb, T, W)), "dt": np.zeros((nb, T, W)), "z": np.zeros((nb, T, W)), "A": np.zeros((W, N)),
         "B": np.zeros((nb, T, G, N)), "C": np.zeros((nb, T, G, N)), "D": np.zeros(W), "dt_bias": np.zeros(W),
         "h_first": np.zeros((nb, W, N)) if grad_last is None else np.array(grad_last, np.float64)}
    for b, n in enumerate(steps(length, nb, T)):
        mu = g["h_first"][b]
        for t in range(n - 1, -1, -1):
            r = dt[b, t] + (0 if dt_bias is None else dt_bias)
            delta, slope = (softplus(r), sigmoid(r)) if softplus_ else (r, 1.0)
            a = np.exp(delta[:, None] * A)
            u = delta * x[b, t]
            h = a * before[b, t] + u[:, None] * B[b, t][of]
            gate = 1.0
            if z is not None:
                s = sigmoid(z[b, t])
                gate = z[b, t] * s
                v = (C[b, t][of] * h).sum(1) + (0 if D is None else D * x[b, t])
                g["z"][b, t] = grad_y[b, t] * v * s * (1 + z[b, t] * (1 - s))
            gg = grad_y[b, t] * gate
            lam = mu + gg[:, None] * C[b, t][of]
            for d in range(W):
                g["C"][b, t, of[d]] += gg[d] * h[d]
                g["B"][b, t, of[d]] += lam[d] * u[d]
            q = lam * a * before[b, t]
            into = (lam * B[b, t][of]).sum(1)
            g["A"] += delta[:, None] * q
            g["dt"][b, t] = ((A * q).sum(1) + x[b, t] * into) * slope
            g["dt_bias"] += g["dt"][b, t]
            g["x"][b, t] = delta * into + (0 if D is None else D * gg)
            g["D"] += gg * x[b, t]
            mu = a * lam
        g["h_first"][b] = mu
    return g
