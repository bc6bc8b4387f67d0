"""Float64 definitions of the operators that run, train and evaluate refined layers.

The gated feed-forward block and its gradients, linear layers in 8-bit
integers, and log probabilities of tokens with their gradient, in NumPy, row by
row where that is the plainest form.
"""

from __future__ import annotations

import math

import numpy as np

_erf = np.vectorize(math.erf, otypes=[np.float64])


def activation(a, act):
    """(act(a), act'(a), a bound on |act'| and |act''|)."""
    a = np.asarray(a, dtype=np.float64)
    if act == "silu":
        with np.errstate(over="ignore"):
            sig = 1.0 / (1.0 + np.exp(-a))
        return a * sig, sig * (1.0 + a * (1.0 - sig)), 1.13
    if act == "gelu":
        cdf = 0.5 * (1.0 + _erf(a / math.sqrt(2.0)))
        return a * cdf, cdf + a * np.exp(-0.5 * a * a) / math.sqrt(2.0 * math.pi), 1.13
    c = math.sqrt(2.0 / math.pi)
    th = np.tanh(c * (a + 0.044715 * a ** 3))
    slope = 0.5 * (1.0 + th) + 0.5 * a * (1.0 - th * th) * c * (1.0 + 3 * 0.044715 * a * a)
    return 0.5 * a * (1.0 + th), slope, 1.13


def gated(X, Wg, Wu, act):
    """(Y, a, b) of Y = act(a) * b, a = X Wg^T, b = X Wu^T."""
    a, b = X @ Wg.T, X @ Wu.T
    return activation(a, act)[0] * b, a, b


def gated_grad(X, Wg, Wu, dY, act):
    """(dX, dWg, dWu, da, db)."""
    a, b = X @ Wg.T, X @ Wu.T
    h, slope, _ = activation(a, act)
    da, db = dY * b * slope, dY * h
    return da @ Wg + db @ Wu, da.T @ X, db.T @ X, da, db


def quant_rows(X):
    """(Q, scale) of fp32 rows: the definition's own fp32 arithmetic."""
    X = np.asarray(X, dtype=np.float32)
    Q = np.zeros(X.shape, dtype=np.int8)
    scale = np.zeros(X.shape[0], dtype=np.float32)
    for r, x in enumerate(X):
        if not np.all(np.isfinite(x)):
            scale[r] = np.nan
            continue
        amax = np.abs(x).max()
        if amax < np.float32(2.0 ** -100):
            continue
        scale[r] = amax / np.float32(127)
        Q[r] = np.rint(x * (np.float32(127) / amax)).astype(np.int8)
    return Q, scale


def matmul_i8(Xq, sx, Wq, sw):
    """(Y, the sum of the groups' magnitudes) for sw [n, G]."""
    k, G = Wq.shape[1], sw.shape[1]
    y = np.zeros((Xq.shape[0], Wq.shape[0]))
    size = np.zeros_like(y)
    for g in range(G):
        cut = slice(g * (k // G), (g + 1) * (k // G))
        part = (Xq[:, cut].astype(np.int64) @ Wq[:, cut].astype(np.int64).T) * sw[:, g].astype(np.float64)
        y += part
        size += np.abs(part)
    s = np.asarray(sx, dtype=np.float64).reshape(-1, 1)
    return s * y, np.abs(s) * size


def logprobs(x, targets, top):
    """(logprob, entropy, lse, top_index, top_logprob) of rows x."""
    T, V = x.shape
    lp, ent, lse = np.zeros(T), np.zeros(T), np.zeros(T)
    idx, val = np.full((T, top), -1, dtype=np.int32), np.full((T, top), np.nan)
    for t in range(T):
        row = np.asarray(x[t], dtype=np.float64)
        if np.any(np.isnan(row)) or np.any(row == np.inf):
            lse[t] = ent[t] = np.nan
            lp[t] = np.nan if targets[t] >= 0 else 0.0
            continue
        live = row[row > -np.inf]
        order = np.lexsort((np.arange(V), -row))[:top]
        idx[t] = order
        if live.size == 0:
            lse[t] = -np.inf
            val[t] = -np.inf
            lp[t] = -np.inf if 0 <= targets[t] < V else 0.0 if targets[t] < 0 else np.nan
            continue
        m = live.max()
        z = np.exp(live - m).sum()
        lse[t] = m + math.log(z)
        ent[t] = math.log(z) - (np.exp(live - m) * (live - m)).sum() / z
        val[t] = row[order] - lse[t]
        if targets[t] >= V:
            lp[t] = np.nan
        elif targets[t] >= 0:
            lp[t] = row[targets[t]] - lse[t]
    return lp, ent, lse, idx, val


def logprobs_grad(x, targets, d_logprob, d_entropy):
    """Gradient of sum(d_logprob logprob + d_entropy entropy) in x."""
    d = np.zeros(x.shape)
    for t, row in enumerate(np.asarray(x, dtype=np.float64)):
        if np.all(row == -np.inf):
            continue
        if np.any(np.isnan(row)) or np.any(row == np.inf) or targets[t] >= len(row):
            d[t] = np.nan
            continue
        m = row.max()
        p = np.exp(row - m)
        p /= p.sum()
        logp = np.log(np.where(p > 0, p, 1.0))
        ent = -(p * logp).sum()
        d[t] = -d_entropy[t] * p * (logp + ent)
        if targets[t] >= 0:
            d[t] -= d_logprob[t] * p
            d[t, targets[t]] += d_logprob[t]
    return d
