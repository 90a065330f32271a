"""The attention block over node states, fp64 (test infrastructure only).

``layer_norm``            y = gamma (x - mean) rstd + beta, with the rows' mean and rstd = (var + eps)^-1/2
``layer_norm_backward``   with xh = (x - mean) rstd, g = gamma dy:
                          dx = rstd (g - mean(g) - xh mean(g xh)), dgamma = sum dy xh, dbeta = sum dy
``linear``                z = x W^T + b, out = act(z) + r
``linear_backward``       dz = dout act'(z), dx = dz W, dW = dz^T x, db = sum dz
``attend``                per query sequence, over the keys of its source that count, per head:
                          s = scale q k^T, p = softmax(s), o = p v, lse = log sum exp s; without a key o = 0, lse = -inf
``attend_backward``       dv = p^T do, dp = do v^T, ds = p (dp - sum p dp), dq = scale ds k, dk = scale ds^T q

From the definitions, one sequence and head at a time.  The product path never imports this module, and it imports nothing
from the product package.
"""
from __future__ import annotations

import math

import numpy as np

_erf = np.vectorize(math.erf, otypes=[np.float64])


def layer_norm(x, gamma=None, beta=None, eps=1e-5):
    x = np.asarray(x, np.float64)
    mean = x.mean(1)
    rstd = 1.0 / np.sqrt(((x - mean[:, None]) ** 2).mean(1) + eps)
    y = (x - mean[:, None]) * rstd[:, None]
    if gamma is not None:
        y = y * np.asarray(gamma, np.float64)
    return (y if beta is None else y + np.asarray(beta, np.float64)), mean, rstd


def layer_norm_backward(x, dy, gamma=None, eps=1e-5, mean=None, rstd=None):
    x, dy = np.asarray(x, np.float64), np.asarray(dy, np.float64)
    if mean is None:
        _, mean, rstd = layer_norm(x, eps=eps)
    xh = (x - np.asarray(mean, np.float64)[:, None]) * np.asarray(rstd, np.float64)[:, None]
    g = dy if gamma is None else dy * np.asarray(gamma, np.float64)
    dx = np.asarray(rstd, np.float64)[:, None] * (g - g.mean(1, keepdims=True) - xh * (g * xh).mean(1, keepdims=True))
    return dx, (dy * xh).sum(0), dy.sum(0)


def activate(act, z):
    z = np.asarray(z, np.float64)
    if act == "relu":
        return np.where(z < 0, 0.0, z)
    if act == "tanh":
        return np.tanh(z)
    return z * 0.5 * (1 + _erf(z / math.sqrt(2))) if act == "gelu" else z


def slope(act, z):
    z = np.asarray(z, np.float64)
    if act == "relu":
        return (z > 0).astype(np.float64)
    if act == "tanh":
        return 1 - np.tanh(z) ** 2
    if act == "gelu":
        return 0.5 * (1 + _erf(z / math.sqrt(2))) + z * np.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    return np.ones_like(z)


def linear(x, W, b=None, act="none", residual=None):
    z = np.asarray(x, np.float64) @ np.asarray(W, np.float64).T
    z = z if b is None else z + np.asarray(b, np.float64)
    out = activate(act, z)
    return (out if residual is None else out + np.asarray(residual, np.float64)), z


def linear_backward(x, W, dout, act="none", z=None):
    dz = np.asarray(dout, np.float64)
    dz = dz if act == "none" else dz * slope(act, z)
    return dz @ np.asarray(W, np.float64), dz.T @ np.asarray(x, np.float64), dz.sum(0), dz


def _pairs(q_ptr, k_ptr, q_rows, k_rows, source, mask):
    """(rows of the queries, rows of the keys that count) of every query sequence that has both."""
    for b in range(len(q_ptr) - 1):
        e = b if source is None else int(source[b])
        at = np.arange(q_ptr[b], q_ptr[b + 1])
        rows = at if q_rows is None else np.asarray(q_rows)[at]
        if e < 0:
            yield rows, np.zeros(0, np.int64)
            continue
        at = np.arange(k_ptr[e], k_ptr[e + 1])
        if mask is not None:
            at = at[np.asarray(mask)[at] != 0]
        yield rows, (at if k_rows is None else np.asarray(k_rows)[at])


def attend(q, k, v, heads, kv_heads, head_dim, q_ptr, k_ptr, q_rows=None, k_rows=None, source=None, mask=None, scale=None):
    """(out [query rows, heads x head_dim], lse [query rows, heads]); rows that no sequence lists are 0 and -inf."""
    scale = head_dim ** -0.5 if scale is None else scale
    q, k, v = (np.asarray(a, np.float64) for a in (q, k, v))
    out, lse = np.zeros((len(q), heads * head_dim)), np.full((len(q), heads), -np.inf)
    for rows, keys in _pairs(q_ptr, k_ptr, q_rows, k_rows, source, mask):
        if len(keys) == 0:
            continue
        for h in range(heads):
            c, g = slice(h * head_dim, (h + 1) * head_dim), h // (heads // kv_heads)
            ck = slice(g * head_dim, (g + 1) * head_dim)
            s = scale * (q[rows, c] @ k[keys, ck].T)
            m = s.max(1, keepdims=True)
            p = np.exp(s - m)
            total = p.sum(1, keepdims=True)
            out[rows, c], lse[rows, h] = (p / total) @ v[keys, ck], (m + np.log(total))[:, 0]
    return out, lse


def attend_backward(q, k, v, dout, heads, kv_heads, head_dim, q_ptr, k_ptr, q_rows=None, k_rows=None, source=None,
                    mask=None, scale=None):
    """(dq, dk, dv); rows that no sequence lists, and keys that do not count, have gradient 0."""
    scale = head_dim ** -0.5 if scale is None else scale
    q, k, v, dout = (np.asarray(a, np.float64) for a in (q, k, v, dout))
    dq, dk, dv = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
    for rows, keys in _pairs(q_ptr, k_ptr, q_rows, k_rows, source, mask):
        if len(keys) == 0:
            continue
        for h in range(heads):
            c, g = slice(h * head_dim, (h + 1) * head_dim), h // (heads // kv_heads)
            ck = slice(g * head_dim, (g + 1) * head_dim)
            s = scale * (q[rows, c] @ k[keys, ck].T)
            p = np.exp(s - s.max(1, keepdims=True))
            p = p / p.sum(1, keepdims=True)
            dp = dout[rows, c] @ v[keys, ck].T
            ds = scale * p * (dp - (p * dp).sum(1, keepdims=True))
            dq[rows, c] += ds @ k[keys, ck]
            dk[np.ix_(keys, range(ck.start, ck.stop))] += ds.T @ q[rows, c]
            dv[np.ix_(keys, range(ck.start, ck.stop))] += p.T @ dout[rows, c]
    return dq, dk, dv
