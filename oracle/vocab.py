"""The vocabulary head over node states, fp64 (test infrastructure only).

``head``            z = s W^T + b for states s [M, H] and W [V, H]
``head_backward``   ds = dz W, dW = dz^T s, db = sum of the rows of dz
``distill``         per row, with q = softmax(t / T) over the teacher's entries (token i_j, logit t_j) that count
                    (token in [0, V), logit above -inf), p^T = softmax(z / T), p = softmax(z) and label y:
                        loss = a T^2 sum_j q_j (log q_j - log p^T[i_j]) - b log p[y]
                        dz_c = scale (a T (p^T_c - sum of q_j over i_j = c) + b (p_c - [c = y]))
``token_logprobs``  log p of given tokens, the entropy -sum p log p, the largest log probabilities (equal ones by the
                    lowest token)

Rows that are no distribution: -inf alone is `empty` (log probabilities -inf, entropy 0; a loss of +inf and no gradient
for a row with a target), NaN or +inf anywhere makes everything of the row NaN.

One row at a time, from the definitions.  The product path never imports this module, and it imports nothing from the
product package.
"""
from __future__ import annotations

import math

import numpy as np


def head(s, W, b=None):
    z = np.asarray(s, np.float64) @ np.asarray(W, np.float64).T
    return z if b is None else z + np.asarray(b, np.float64)


def head_backward(s, W, dz):
    s, W, dz = (np.asarray(a, np.float64) for a in (s, W, dz))
    return dz @ W, dz.T @ s, dz.sum(axis=0)


def _log_softmax(z):
    """log p of one row that holds a largest finite value."""
    m = z.max()
    with np.errstate(over="ignore"):
        d = z - m
    return d - math.log(np.exp(d).sum())


def _kind(z):
    if np.isnan(z).any() or (z == np.inf).any():
        return "bad"
    return "empty" if (z == -np.inf).all() else "fine"


def distill(z, tok=None, t=None, y=None, T=1.0, soft=1.0, hard=0.0, scale=1.0):
    """(losses [M], dz [M, V]) for logits z [M, V], tok and t [M, k], y [M]."""
    z = np.asarray(z, np.float64)
    M, V = z.shape
    loss, dz = np.zeros(M), np.zeros((M, V))
    for r in range(M):
        ent = [] if tok is None else [(int(i), float(v)) for i, v in zip(tok[r], t[r]) if 0 <= i < V and v != -np.inf]
        lab = -1 if y is None or not 0 <= y[r] < V else int(y[r])
        if not ent and lab < 0:
            continue
        kind = _kind(z[r])
        if kind != "fine":
            loss[r] = np.nan if kind == "bad" else np.inf
            dz[r] = np.nan if kind == "bad" else 0.0
            continue
        if ent:
            tv = np.array([v for _, v in ent])
            lq = _log_softmax(tv / T)
            lp = _log_softmax(z[r] / T)
            dz[r] += scale * soft * T * np.exp(lp)
            for (i, _), l in zip(ent, lq):
                q = math.exp(l)
                if q > 0 and soft > 0:
                    loss[r] += soft * T * T * q * (l - lp[i])
                dz[r, i] -= scale * soft * T * q
        if lab >= 0 and hard > 0:
            lp = _log_softmax(z[r])
            loss[r] -= hard * lp[lab]
            dz[r] += scale * hard * np.exp(lp)
            dz[r, lab] -= scale * hard
    return loss, dz


def token_logprobs(z, tokens, K=0):
    """(logp [M, J], entropy [M], top_token [M, K], top_logp [M, K])."""
    z = np.asarray(z, np.float64)
    M, V = z.shape
    tokens = np.asarray(tokens)
    logp, ent = np.zeros(tokens.shape), np.zeros(M)
    top, top_lp = np.full((M, K), -1, np.int64), np.full((M, K), -np.inf)
    for r in range(M):
        kind = _kind(z[r])
        lp = (_log_softmax(z[r]) if kind == "fine" else np.full(V, np.nan if kind == "bad" else -np.inf))
        for j, i in enumerate(tokens[r]):
            logp[r, j] = lp[i] if 0 <= i < V else 0.0
        if kind == "bad":
            ent[r], top_lp[r] = np.nan, np.nan
            continue
        p = np.exp(lp)
        ent[r] = -(p[p > 0] * lp[p > 0]).sum()
        order = [c for c in np.lexsort((np.arange(V), -z[r]))[:K] if z[r, c] > -np.inf]
        top[r, :len(order)] = order
        top_lp[r, :len(order)] = lp[order]
    return logp, ent, top, top_lp
