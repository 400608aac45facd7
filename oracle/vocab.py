"""The operators at the vocabulary's two ends of a packed step, by their
definitions in float64: the embedding of its tokens, log probabilities of the
targets from the last hidden rows, and the divergence from a teacher's top
alternatives; each with its gradient.  Plain numpy on whole arrays; see
include/nsp.h for the conventions.
"""
from __future__ import annotations

import numpy as np

from . import rows as R


def linear_logp(x, w, targets, scale=1.0):
    """dict of logp, lse, entropy of the logits x w^T."""
    z = np.asarray(x, np.float64) @ np.asarray(w, np.float64).T
    return R.token_logp(z, targets, scale)


def linear_logp_backward(x, w, targets, lse, entropy, g_logp=None, g_lse=None, g_entropy=None, scale=1.0):
    """(dx, dw, gradient of the logits) for the lse and entropy given.  Tokens without a
    gradient take no part, whatever their rows hold."""
    x, w = np.asarray(x, np.float64), np.asarray(w, np.float64)
    y = None if targets is None else np.asarray(targets)
    live = np.asarray(lse, np.float64) != -np.inf
    g = np.zeros(len(x), bool)
    if g_logp is not None:
        g |= (np.asarray(g_logp) != 0) & (y >= 0) & (y < len(w))
    for more in (g_lse, g_entropy):
        if more is not None:
            g |= np.asarray(more) != 0
    live &= g
    xs = np.where(live[:, None], x, 0.0)
    da = R.token_logp_backward(xs @ w.T, y, lse, entropy, g_logp, g_lse, g_entropy, scale)
    da[~live] = 0.0
    return da @ w, da.T @ xs, da


def weights(index, teacher, vocab, normalized=False):
    """q [T, top] and t - c, zeros where there is no alternative, and which are one."""
    index, t = np.asarray(index), np.asarray(teacher, np.float64)
    with np.errstate(invalid="ignore"):
        there = (index >= 0) & (index < vocab) & ~(t <= R.MASKED)
    q, d = np.zeros(t.shape), np.zeros(t.shape)
    for r in range(len(t)):
        v = t[r, there[r]]
        if not len(v):
            continue
        if np.isnan(v).any() or (v == np.inf).any():
            q[r], d[r] = np.nan, np.nan
            continue
        c = v.max() + np.log(np.exp(v - v.max()).sum()) if normalized else 0.0
        d[r, there[r]] = v - c
        q[r, there[r]] = np.exp(v - c)
    return q, d, there


def distill(logits, index, teacher, normalized=False, scale=1.0):
    """(loss, lse)."""
    raw = np.asarray(logits, np.float64)
    T, V = raw.shape
    lse = R.token_logp(raw, np.full(T, -1), scale)["lse"]
    q, d, there = weights(index, teacher, V, normalized)
    loss = np.zeros(T)
    for t in range(T):
        if not there[t].any():
            continue
        if np.isnan(lse[t]) or np.isnan(q[t]).any():
            loss[t] = np.nan
            continue
        for k in np.flatnonzero(there[t] & (q[t] > 0)):
            z = raw[t, index[t, k]]
            lp = -np.inf if z <= R.MASKED or lse[t] == -np.inf else z * scale - lse[t]
            loss[t] += q[t, k] * (d[t, k] - lp)
    return loss, lse


def distill_backward(logits, index, teacher, lse, g, normalized=False, scale=1.0):
    """Gradient of the logits for the lse given (p at most 1)."""
    raw = np.asarray(logits, np.float64)
    T, V = raw.shape
    q, _, there = weights(index, teacher, V, normalized)
    out = np.zeros((T, V))
    for t in range(T):
        if not there[t].any() or g[t] == 0 or lse[t] == -np.inf:
            continue
        if np.isnan(q[t]).any():
            out[t] = np.nan
            continue
        out[t] = np.exp(np.minimum(raw[t] * scale - float(lse[t]), 0.0)) * q[t].sum()
        np.subtract.at(out[t], index[t, there[t]], q[t, there[t]])
        out[t] *= float(g[t])
    return out * scale


def embedding(tokens, w, scale=1.0):
    tokens, w = np.asarray(tokens), np.asarray(w, np.float64)
    y = np.zeros((len(tokens), w.shape[1]))
    for t, v in enumerate(tokens):
        if 0 <= v < len(w):
            y[t] = scale * w[v]
    return y


def embedding_backward(tokens, dy, vocab, scale=1.0):
    tokens, dy = np.asarray(tokens), np.asarray(dy, np.float64)
    dw = np.zeros((vocab, dy.shape[1]))
    for t, v in enumerate(tokens):
        if 0 <= v < vocab:
            dw[v] += dy[t]
    return scale * dw
