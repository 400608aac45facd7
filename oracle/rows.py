"""Row operators around the attention, by their definitions in float64.

Rotary positions (Background, Sequence Packing: position ids restart at every
packed sequence), norms of rows, and the log probabilities of given tokens
with entropy and top alternatives; each with its gradient.  Plain numpy on
whole arrays; see include/nsp.h for the conventions.
"""
from __future__ import annotations

import numpy as np

MASKED = -2.0 ** 126                 # logits up to here are a masked vocabulary


def rotary(x, positions, freqs, pairs=False, scale=1.0, backward=False):
    """x [T, H, D] turned by positions [T] x freqs [r / 2]."""
    x = np.asarray(x, np.float64)
    r = 2 * len(freqs)
    a = np.asarray(positions, np.float64)[:, None, None] * np.asarray(freqs, np.float64)
    c, s = scale * np.cos(a), scale * np.sin(a)
    if backward:
        s = -s
    first, second = (slice(0, r, 2), slice(1, r, 2)) if pairs else (slice(0, r // 2), slice(r // 2, r))
    y = x.copy()
    y[..., first] = x[..., first] * c - x[..., second] * s
    y[..., second] = x[..., second] * c + x[..., first] * s
    return y


def norm(x, w=None, b=None, eps=0.0, rms=False):
    """(y, mean, rstd) of the rows of x [..., n]."""
    x = np.asarray(x, np.float64)
    mean = np.zeros(x.shape[:-1]) if rms else x.mean(-1)
    d = x - mean[..., None]
    rstd = 1.0 / np.sqrt((d * d).mean(-1) + eps)
    y = d * rstd[..., None]
    y = y if w is None else y * w
    return (y if b is None else y + b), mean, rstd


def norm_backward(x, w, dy, mean, rstd, rms=False):
    """(dx, dw, db) for the statistics given."""
    x, dy = np.asarray(x, np.float64), np.asarray(dy, np.float64)
    n = x.shape[-1]
    xh = (x - (0.0 if rms else np.asarray(mean, np.float64)[..., None])) * np.asarray(rstd, np.float64)[..., None]
    h = dy if w is None else dy * w
    dx = h - xh * (h * xh).mean(-1, keepdims=True)
    if not rms:
        dx -= h.mean(-1, keepdims=True)
    dx *= np.asarray(rstd, np.float64)[..., None]
    return dx, (dy * xh).reshape(-1, n).sum(0), dy.reshape(-1, n).sum(0)


def token_logp(logits, targets, scale=1.0, top=0):
    """dict of logp, lse, entropy, top_logp, top_index of logits [T, V]."""
    raw = np.asarray(logits, np.float64)
    T, V = raw.shape
    out = {"logp": np.zeros(T), "lse": np.zeros(T), "entropy": np.zeros(T), "top_logp": np.full((T, top), -np.inf),
           "top_index": np.full((T, top), -1, np.int64)}
    for t in range(T):
        z = np.where(raw[t] <= MASKED, -np.inf, raw[t]) * scale
        y = int(targets[t])
        given = 0 <= y < V
        if np.isnan(z).any() or (z == np.inf).any():
            lse = ent = np.nan
        elif (z == -np.inf).all():
            lse, ent = -np.inf, 0.0
        else:
            lse = z.max() + np.log(np.exp(z - z.max()).sum())
            p = np.exp(z - lse)
            ent = lse - (p[p > 0] * z[p > 0]).sum()
        out["lse"][t], out["entropy"][t] = lse, ent
        if given:
            out["logp"][t] = -np.inf if lse == -np.inf else z[y] - lse
        order = [v for v in np.lexsort((np.arange(V), -np.where(np.isnan(raw[t]), -np.inf, raw[t])))[:top]
                 if raw[t, v] > MASKED]
        out["top_index"][t, :len(order)] = order
        out["top_logp"][t, :len(order)] = z[order] - lse
    return out


def token_logp_backward(logits, targets, lse, entropy, g_logp=None, g_lse=None, g_entropy=None, scale=1.0):
    """Gradient of the logits for the lse and entropy given."""
    raw = np.asarray(logits, np.float64)
    T, V = raw.shape
    out = np.zeros((T, V))
    for t in range(T):
        y = -1 if targets is None else int(targets[t])
        gl = 0.0 if g_logp is None or not 0 <= y < V else float(g_logp[t])
        gs = 0.0 if g_lse is None else float(g_lse[t])
        ge = 0.0 if g_entropy is None else float(g_entropy[t])
        if lse[t] == -np.inf or (gl == 0 and gs == 0 and ge == 0):
            continue
        d = raw[t] * scale - float(lse[t])
        p = np.exp(d)
        out[t] = (gs - gl) * p
        if ge != 0:
            live = p > 0
            out[t, live] -= ge * p[live] * (d[live] + float(entropy[t]))
        if gl != 0:
            out[t, y] += gl
    return out * scale
