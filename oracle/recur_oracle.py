"""Plain fp64 CPU oracle for the channel-wise gated recurrence, with its gradients
and the bounds that its roundings leave.

TEST INFRASTRUCTURE ONLY, as oracle/vda_oracle.py: straight from the
definitions, one token at a time, sharing nothing with the HIP library.

    h_t = a_t h_{t-1} + u_t,  out_t = h_t,
    log: a = e^g, u = x;  logit: a = 1 / (1 + e^-g), u = (1 - a) x;  norm: a likewise, u = sqrt(1 - a^2) x.
"""
from __future__ import annotations

import numpy as np


def _parts(g, gate):
    """a, 1 - a, the weight of x, and both weights' derivatives by g."""
    if gate == "log":
        a = np.exp(g)
        return a, -np.expm1(g), np.ones_like(g), a, np.zeros_like(g)
    with np.errstate(over="ignore"):
        a, b = 1 / (1 + np.exp(-g)), 1 / (1 + np.exp(g))
    if gate == "logit":
        return a, b, b, a * b, -a * b
    return a, b, np.sqrt(b * (1 + a)), a * b, -a * a * np.sqrt(b / (1 + a))


def recur_sequence(x, g, gate, h, reverse=False):
    """x, g [L, C], h [C] -> out [L, C], the last state."""
    a, _, w, _, _ = _parts(g, gate)
    out, h = np.zeros_like(x), h.copy()
    for t in (reversed(range(len(x))) if reverse else range(len(x))):
        h = np.where(a[t] == 0, 0.0, a[t] * h) + w[t] * x[t]
        out[t] = h
    return out, h


def recur_sequence_backward(do, dS, x, g, gate, h, reverse=False):
    """Gradients of recur_sequence: dx, dg, dh."""
    a, _, w, da, dw = _parts(g, gate)
    order = list(range(len(x)))[::-1] if reverse else list(range(len(x)))
    before, s = np.zeros_like(x), h.copy()
    for t in order:
        before[t] = s
        s = a[t] * s + w[t] * x[t]
    dx, dg, D = np.zeros_like(x), np.zeros_like(x), dS.copy()
    for t in reversed(order):
        D = D + do[t]
        dx[t] = w[t] * D
        dg[t] = D * (da[t] * before[t] + dw[t] * x[t])
        D = a[t] * D
    return dx, dg, D


def recur_bounds(x, g, gate, h, half, reverse=False, do=None, dS=None):
    """How far each output may be off by its roundings: (out, state) or (dx, dg, dh).

    f = 2^-24 a rounding's relative error to fp32, `half` to the storage type.  A gate's power of two
    has its argument rounded (|g| f) and 2 f of its own, a reciprocal 2 f, a square root 2 f: a, 1 - a
    and the weight have relative errors of k = (|g| + 8) f.  A step multiplies and adds, 2 f; a
    tile's product of decays multiplies at most two more than that: c = 3 (k + 2 f) of the sizes that
    enter each step covers them.
    """
    f = 2.0 ** -24
    a, _, w, da, dw = _parts(g, gate)
    c = 3 * (np.minimum(np.abs(g), 100.0) + 10) * f
    order = list(range(len(x)))[::-1] if reverse else list(range(len(x)))
    size, err = np.abs(h), np.zeros_like(h)  # of the state: the sum of magnitudes, the error
    size_b, err_b, e_out = np.zeros_like(x), np.zeros_like(x), np.zeros_like(x)
    out, _ = recur_sequence(x, g, gate, h, reverse)
    for t in order:
        size_b[t], err_b[t] = size, err
        err = a[t] * err + c[t] * (a[t] * size + w[t] * np.abs(x[t]))
        size = a[t] * size + w[t] * np.abs(x[t])
        e_out[t] = err + half * np.abs(out[t])
    if do is None:
        return e_out, err
    dx, dg, _ = recur_sequence_backward(do, dS, x, g, gate, h, reverse)
    e_dx, e_dg = np.zeros_like(x), np.zeros_like(x)
    D, eD = np.abs(dS), np.zeros_like(dS)
    for t in reversed(order):
        D = D + np.abs(do[t])
        eD = eD + c[t] * D
        e_dx[t] = w[t] * eD + c[t] * w[t] * D + half * np.abs(dx[t])
        parts = np.abs(da[t]) * size_b[t] + np.abs(dw[t]) * np.abs(x[t])
        e_dg[t] = eD * parts + D * (np.abs(da[t]) * err_b[t] + 3 * c[t] * parts) + half * np.abs(dg[t])
        eD = a[t] * eD + c[t] * a[t] * D
        D = a[t] * D
    return e_dx, e_dg, eD
