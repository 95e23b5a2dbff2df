"""Plain fp64 CPU oracle for the token-wise gated delta rule (Eq. 2) and the
multi-axis rotary positions, with their gradients.

TEST INFRASTRUCTURE ONLY, as oracle/vda_oracle.py: straight from the
definitions, one token and one head at a time, sharing nothing with the HIP
library.

The rule, per value head and token in order, on a state S [d_v, d_k]:
    Sbar = exp(g) S,  e = v - Sbar k,  S = Sbar + beta e k^T,  o = scale S q.
Its gradients are the reverse recurrence of these four assignments.
"""
from __future__ import annotations

import numpy as np


def delta_head(q, k, v, g, beta, S, scale):
    """q, k [L, d_k], v [L, d_v], g, beta [L], S [d_v, d_k] -> o [L, d_v], S."""
    o = np.zeros_like(v)
    S = S.copy()
    for t in range(len(g)):
        S = np.exp(g[t]) * S
        e = v[t] - S @ k[t]
        S = S + beta[t] * np.outer(e, k[t])
        o[t] = scale * (S @ q[t])
    return o, S


def delta_head_backward(do, dS, q, k, v, g, beta, S, scale):
    """Gradients of delta_head: (dq, dk, dv, dg, dbeta, dS_in)."""
    L = len(g)
    before = []
    for t in range(L):
        before.append(S)
        S = np.exp(g[t]) * S
        S = S + beta[t] * np.outer(v[t] - S @ k[t], k[t])
    dq, dk, dv = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
    dg, db = np.zeros(L), np.zeros(L)
    dS = dS.copy()
    for t in reversed(range(L)):
        Sbar = np.exp(g[t]) * before[t]
        e = v[t] - Sbar @ k[t]
        S = Sbar + beta[t] * np.outer(e, k[t])
        dq[t] = scale * (S.T @ do[t])
        dS = dS + scale * np.outer(do[t], q[t])
        # S = Sbar + beta e k^T
        de = beta[t] * (dS @ k[t])
        db[t] = e @ (dS @ k[t])
        dk[t] = beta[t] * (dS.T @ e)
        # e = v - Sbar k
        dv[t] = de
        dk[t] -= Sbar.T @ de
        dSbar = dS - np.outer(de, k[t])
        dg[t] = np.sum(dSbar * Sbar)
        dS = np.exp(g[t]) * dSbar
    return dq, dk, dv, dg, db, dS


def delta_sequences(q, k, v, g, beta, cu, S_in, scale):
    """Heads layout over packed sequences: q, k [H_k, T, d_k], v [H_v, T, d_v],
    g, beta [H_v, T], S_in [n, H_v, d_v, d_k] or None; rows outside every
    sequence are NaN in the output."""
    Hv, group, n = v.shape[0], v.shape[0] // q.shape[0], len(cu) - 1
    out = np.full(v.shape, np.nan)
    S = np.zeros((n, Hv, v.shape[2], q.shape[2])) if S_in is None else S_in.copy()
    for i in range(n):
        s = slice(cu[i], cu[i + 1])
        for h in range(Hv):
            out[h, s], S[i, h] = delta_head(q[h // group, s], k[h // group, s], v[h, s], g[h, s],
                                            beta[h, s], S[i, h], scale)
    return out, S


def delta_sequences_backward(do, dS_out, q, k, v, g, beta, cu, S_in, scale):
    """Gradients of delta_sequences; rows outside every sequence are NaN."""
    Hv, group, n = v.shape[0], v.shape[0] // q.shape[0], len(cu) - 1
    shape = (n, Hv, v.shape[2], q.shape[2])
    S = np.zeros(shape) if S_in is None else S_in
    dS = np.zeros(shape) if dS_out is None else dS_out.copy()
    dq, dk, dv, dg, db = (np.full(x.shape, np.nan) for x in (q, k, v, g, beta))
    for i in range(n):
        s = slice(cu[i], cu[i + 1])
        dq[:, s] = dk[:, s] = 0.0
        for h in range(Hv):
            r = delta_head_backward(do[h, s], dS[i, h], q[h // group, s], k[h // group, s], v[h, s],
                                    g[h, s], beta[h, s], S[i, h], scale)
            dq[h // group, s] += r[0]
            dk[h // group, s] += r[1]
            dv[h, s], dg[h, s], db[h, s], dS[i, h] = r[2:]
    return dq, dk, dv, dg, db, dS


def rope_turns(positions, inv_freq, axes):
    """cos and sin [L, R] of the pairs' angles, positions [L, 3]."""
    axis = np.repeat(np.arange(3), axes)
    a = positions[:, axis].astype(np.float64) * inv_freq.astype(np.float64)
    return np.cos(a), np.sin(a)


def _pair_channels(R, interleaved):
    p = np.arange(R)
    return (2 * p, 2 * p + 1) if interleaved else (p, R + p)


def rope_head(x, positions, inv_freq, axes, interleaved, l2):
    """x [L, d] of one head -> its rotation [L, d]."""
    if l2:
        x = x / np.sqrt(np.sum(x * x, -1, keepdims=True) + 1e-6)
    c, s = rope_turns(positions, inv_freq, axes)
    a, b = _pair_channels(int(np.sum(axes)), interleaved)
    y = x.copy()
    y[:, a] = x[:, a] * c - x[:, b] * s
    y[:, b] = x[:, a] * s + x[:, b] * c
    return y


def rope_head_backward(dy, x, positions, inv_freq, axes, interleaved, l2):
    c, s = rope_turns(positions, inv_freq, axes)
    a, b = _pair_channels(int(np.sum(axes)), interleaved)
    dx = dy.copy()
    dx[:, a] = dy[:, a] * c + dy[:, b] * s
    dx[:, b] = dy[:, b] * c - dy[:, a] * s
    if l2:
        n = np.sqrt(np.sum(x * x, -1, keepdims=True) + 1e-6)
        dx = dx / n - x * np.sum(x * dx, -1, keepdims=True) / n ** 3
    return dx


def grid_positions(L, grid_h, grid_w, frame_offset):
    i = np.arange(L)
    return np.stack([frame_offset + i // (grid_h * grid_w), i // grid_w % grid_h, i % grid_w], -1)
