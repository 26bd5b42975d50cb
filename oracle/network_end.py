"""Layer norm, log probabilities and the distillation loss in numpy's 64-bit floats, written from their definitions, a row
at a time where a row can be out of the ordinary.  Inputs of any float type are taken as the values they hold."""
from __future__ import annotations

import numpy as np


# ---------------------------------------------------------------- layer norm
def layer_norm_forward(x, gamma=None, beta=None, eps=1e-5):
    """(y, mean, rstd) over the last axis."""
    x = np.asarray(x, dtype=np.float64)
    mean = x.mean(axis=-1)
    rstd = 1.0 / np.sqrt(((x - mean[..., None]) ** 2).mean(axis=-1) + eps)
    y = (x - mean[..., None]) * rstd[..., None]
    if gamma is not None:
        y = y * np.asarray(gamma, dtype=np.float64)
    if beta is not None:
        y = y + np.asarray(beta, dtype=np.float64)
    return y, mean, rstd


def layer_norm_backward(x, dy, mean, rstd, gamma=None):
    """(dx, dgamma, dbeta) for the statistics given."""
    x, dy = np.asarray(x, dtype=np.float64), np.asarray(dy, dtype=np.float64)
    mean, rstd = np.asarray(mean, dtype=np.float64)[..., None], np.asarray(rstd, dtype=np.float64)[..., None]
    xh = (x - mean) * rstd
    g = dy if gamma is None else dy * np.asarray(gamma, dtype=np.float64)
    dx = rstd * (g - g.mean(axis=-1, keepdims=True) - xh * (g * xh).mean(axis=-1, keepdims=True))
    lead = tuple(range(x.ndim - 1))
    return dx, (dy * xh).sum(axis=lead), dy.sum(axis=lead)


# ---------------------------------------------------------------- softmax of a row
def log_softmax_row(x, temperature=1.0):
    """ln p of one row.  No possible class: -inf everywhere.  A NaN or +inf: NaN everywhere."""
    x = np.asarray(x, dtype=np.float64)
    if np.any(np.isnan(x)) or np.any(x == np.inf):
        return np.full(x.shape, np.nan)
    m = x.max()
    if m == -np.inf:
        return np.full(x.shape, -np.inf)
    z = (x - m) / temperature
    return z - np.log(np.exp(z).sum())


def logprob_forward(logits, targets=None, top=0, temperature=1.0):
    """(logprob, entropy, top_index, top_logprob) of logits [rows][classes], targets [rows][given]."""
    logits = np.asarray(logits, dtype=np.float64)
    rows, n = logits.shape
    given = 0 if targets is None else targets.shape[1]
    logprob, entropy = np.zeros((rows, given)), np.zeros(rows)
    index, best = np.full((rows, top), -1, dtype=np.int64), np.full((rows, top), -np.inf)
    for r in range(rows):
        lp = log_softmax_row(logits[r], temperature)
        p = np.exp(lp)
        there = p > 0
        entropy[r] = np.nan if np.isnan(lp).any() else -(p[there] * lp[there]).sum()
        for j in range(given):
            t = targets[r, j]
            logprob[r, j] = 0.0 if t < 0 else (np.nan if t >= n else lp[t])
        # descending, equal values by ascending index; -inf and NaN are nobody's alternatives
        possible = np.nonzero(logits[r] > -np.inf)[0] if top else np.zeros(0, dtype=np.int64)
        if possible.size > top:   # only those that reach the top-th largest are put in order
            possible = possible[logits[r, possible] >= np.partition(logits[r, possible], -top)[-top]] if top else possible[:0]
        order = possible[np.lexsort((possible, -logits[r, possible]))][:top]
        index[r, :len(order)] = order
        best[r, :len(order)] = lp[order]
    return logprob, entropy, index, best


def logprob_backward(logits, targets, dlogprob, dentropy=None, temperature=1.0):
    logits = np.asarray(logits, dtype=np.float64)
    rows, n = logits.shape
    out = np.zeros((rows, n))
    for r in range(rows):
        lp = log_softmax_row(logits[r], temperature)
        if np.isnan(lp).any() or (targets is not None and (targets[r] >= n).any()):
            out[r] = np.nan
            continue
        if lp.max() == -np.inf:
            continue
        p = np.exp(lp)
        finite = np.where(p > 0, lp, 0.0)
        if dentropy is not None:
            out[r] -= dentropy[r] * p * (finite - (p * finite).sum())
        for j in range(0 if targets is None else targets.shape[1]):
            if targets[r, j] >= 0:
                out[r] -= dlogprob[r, j] * p
                out[r, targets[r, j]] += dlogprob[r, j]
    return out / temperature


# ---------------------------------------------------------------- distillation
def distill(logits, index=None, teacher=None, labels=None, temperature=1.0, alpha=1.0, w=None):
    """(loss [rows], gradient [rows][classes] of sum(w * loss))."""
    logits = np.asarray(logits, dtype=np.float64)
    rows, n = logits.shape
    loss, grad = np.zeros(rows), np.zeros((rows, n))
    w = np.ones(rows) if w is None else np.asarray(w, dtype=np.float64)
    for r in range(rows):
        lp, lp1 = log_softmax_row(logits[r], temperature), log_softmax_row(logits[r])
        none = lp.max() == -np.inf
        if index is not None and alpha > 0:
            at, t = np.asarray(index[r]), np.asarray(teacher[r], dtype=np.float64)
            there = (at >= 0) & (t != -np.inf)
            at, t = at[there], t[there]
            if at.size and ((at >= n).any() or not np.isfinite(t).all()):
                loss[r], grad[r] = np.nan, np.nan
                continue
            if at.size:
                lnq = log_softmax_row(t, temperature)
                q = np.exp(lnq)
                for k in range(at.size):
                    if q[k] > 0:
                        loss[r] += alpha * temperature ** 2 * q[k] * (lnq[k] - lp[at[k]])
                if not none:
                    g = np.exp(lp)
                    np.subtract.at(g, at, q)
                    grad[r] += w[r] * alpha * temperature * g
        if labels is not None and alpha < 1 and labels[r] >= 0:
            if labels[r] >= n:
                loss[r], grad[r] = np.nan, np.nan
                continue
            loss[r] += (1 - alpha) * -lp1[labels[r]]
            if not none:
                g = np.exp(lp1)
                g[labels[r]] -= 1.0
                grad[r] += w[r] * (1 - alpha) * g
    return loss, grad
