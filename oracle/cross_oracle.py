"""Plain fp64 CPU oracle for the cross attention to an encoder's states, with its
gradients and the bounds that its roundings leave.

TEST INFRASTRUCTURE ONLY, as oracle/vda_oracle.py: straight from the
definitions, one sequence and one head at a time, sharing nothing with the HIP
library.

Per row q and the states that are seen:
    s_j = scale q.k_j,  lse = log sum_j e^s_j,  out = sum_j e^(s_j - lse) v_j,
a row that sees none has out = 0 and lse = -inf.
"""
from __future__ import annotations

import numpy as np


def cross_head(q, k, v, scale):
    """q [L, d], k, v [S, d] (the states that are seen) -> out [L, d], lse [L], weights [L, S]."""
    if k.shape[0] == 0:
        return np.zeros_like(q), np.full(q.shape[0], -np.inf), np.zeros((q.shape[0], 0))
    s = scale * (q @ k.T)
    top = s.max(-1, keepdims=True)
    e = np.exp(s - top)
    total = e.sum(-1, keepdims=True)
    p = e / total
    return p @ v, (top + np.log(total))[:, 0], p


def cross_head_backward(do, q, k, v, scale):
    """Gradients of cross_head: dq, dk, dv."""
    out, _, p = cross_head(q, k, v, scale)
    dp = do @ v.T
    ds = p * (dp - (do * out).sum(-1, keepdims=True))
    return scale * (ds @ k), scale * (ds.T @ q), p.T @ do


def cross_sequence(q, k, v, seen, scale, do=None):
    """q [L, H_q, d], k, v [S, H_k, d], seen [S] bool -> out, lse [L, H_q], and with do: dq, dk, dv."""
    group = q.shape[1] // k.shape[1]
    out, lse = np.zeros_like(q), np.zeros(q.shape[:2])
    dq, dk, dv = np.zeros_like(q), np.zeros(k.shape), np.zeros(v.shape)
    for h in range(q.shape[1]):
        kh, vh = k[seen, h // group], v[seen, h // group]
        out[:, h], lse[:, h], _ = cross_head(q[:, h], kh, vh, scale)
        if do is not None and len(kh):
            a, b, c = cross_head_backward(do[:, h], q[:, h], kh, vh, scale)
            dq[:, h] = a
            dk[seen, h // group] += b
            dv[seen, h // group] += c
    return (out, lse) if do is None else (out, lse, dq, dk, dv)


def cross_bounds(q, k, v, seen, scale, half, do=None):
    """How far each output may be off by its roundings, element by element.

    `half`: the largest relative error of a rounding to the storage type; f = 2^-24 that of one to
    fp32.  With A_j = sum_c |q_c k_c| |scale|:
    * a score is a sum of d products, then one product and one difference with the maximum (a number
      of at most max |s|) in fp32, and its power of two has an error of 2 f:
      a weight's relative error is e = max_j ((d + 4) f A_j) + (2 max |s| + 4) f, twice that with its
      sum's, plus S f from the sum's additions, where every term is positive;
    * a weight is rounded to the storage type once where it enters a product, which adds S products;
    * the output is rounded once.
    The gradients take dP_j (a sum of d products, (d + 2) f sum |do v_j|), D (do times the stored
    output, with that output's error), and dS_j, rounded to the storage type once, into sums over S
    states or all rows that share the key head.  bf16 only: the storage roundings (fp32 storage has
    half = f throughout).
    """
    f = 2.0 ** -24
    L, Hq, d = q.shape
    group, S = Hq // k.shape[1], int(seen.sum())
    b_out, b_lse = np.zeros_like(q), np.zeros((L, Hq))
    b_dq, b_dk, b_dv = np.zeros_like(q), np.zeros(k.shape), np.zeros(v.shape)
    for h in range(Hq):
        hk = h // group
        kh, vh = k[seen, hk], v[seen, hk]
        if S == 0 or L == 0:
            continue
        out, lse, p = cross_head(q[:, h], kh, vh, scale)
        A = abs(scale) * (np.abs(q[:, h]) @ np.abs(kh).T)
        e = ((d + 4) * f * A.max(-1) + (2 * (np.abs(scale * (q[:, h] @ kh.T)).max(-1) + 8) + 4) * f)[:, None]
        w = p @ np.abs(vh)
        b_out[:, h] = (2 * e + 2 * S * f + half) * w + half * np.abs(out)
        b_lse[:, h] = (e[:, 0] + S * f) + 2 * f * (np.abs(lse) + 8)
        if do is None:
            continue
        g = do[:, h]
        dp = g @ vh.T
        D = (g * out).sum(-1, keepdims=True)
        ds = p * (dp - D)
        e_p = e + (b_lse[:, h])[:, None]  # the weight is made from the stored lse
        e_d = (np.abs(g) * b_out[:, h]).sum(-1, keepdims=True) + d * f * (np.abs(g) * np.abs(out)).sum(-1, keepdims=True)
        e_ds = p * (2 * e_p * np.abs(dp - D) + (d + 2) * f * (np.abs(g) @ np.abs(vh).T) + e_d) + half * np.abs(ds)
        rows = L * group
        b_dq[:, h] = abs(scale) * (e_ds @ np.abs(kh) + (S + 2) * f * (np.abs(ds) @ np.abs(kh)))
        b_dk[seen, hk] += abs(scale) * (e_ds.T @ np.abs(q[:, h]) + (rows + 2) * f * (np.abs(ds).T @ np.abs(q[:, h])))
        b_dv[seen, hk] += ((2 * e_p + half + (rows + 2) * f) * p).T @ np.abs(g)
    if do is None:
        return b_out, b_lse
    _, _, dq, dk, dv = cross_sequence(q, k, v, seen, scale, do)
    return (b_out, b_lse, b_dq + half * np.abs(dq), b_dk + half * np.abs(dk), b_dv + half * np.abs(dv))
