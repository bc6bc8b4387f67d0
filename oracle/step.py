"""Float64 definitions of the operators around a block in a training or serving step.

The root-mean-square norm (its 8-bit form in the definition's own fp32 arithmetic) and its
gradients, log probabilities from hidden states with their gradients, and AdamW with
its moments in 32 or 8 bits, in NumPy.
"""

from __future__ import annotations

import numpy as np

F = np.float32


def norm(H, gain, eps):
    """(Y, r) of rows H."""
    r = 1.0 / np.sqrt(np.mean(H * H, axis=1, keepdims=True) + eps)
    return H * r * gain, r


def norm_i8(H, gain, eps):
    """(Q, scale) of rows H and gain as fp32: the integers in fp32, the scale in 64 bits."""
    H, gain = np.asarray(H, dtype=F), np.asarray(gain, dtype=F)
    Q = np.zeros(H.shape, dtype=np.int8)
    scale = np.zeros(len(H))
    for t, h in enumerate(H):
        with np.errstate(over="ignore", invalid="ignore"):
            w = h * gain
        if not np.all(np.isfinite(w)):
            scale[t] = np.nan
            continue
        amax = np.abs(w).max()
        if amax < F(2.0 ** -100):
            continue
        Q[t] = np.rint(w * (F(127) / amax)).astype(np.int8)
        scale[t] = float(amax) / 127.0 / np.sqrt(np.mean(h.astype(np.float64) ** 2) + eps)
    return Q, scale


def norm_grad(H, gain, dY, dH, eps):
    """(dX, dgain)."""
    r = norm(H, gain, eps)[1]
    u = dY * gain
    dx = r * u - H * r ** 3 * np.mean(u * H, axis=1, keepdims=True)
    return dx + (0.0 if dH is None else dH), (dY * H * r).sum(axis=0)


def linear_logprobs(X, W, targets):
    """(logprob, lse, p)."""
    logits = X @ W.T
    m = logits.max(axis=1)
    e = np.exp(logits - m[:, None])
    lse = m + np.log(e.sum(axis=1))
    lp = np.zeros(len(X))
    for t, v in enumerate(targets):
        if v >= len(W):
            lp[t] = np.nan
        elif v >= 0:
            lp[t] = logits[t, v] - lse[t]
    return lp, lse, e / e.sum(axis=1, keepdims=True)


def linear_logprobs_grad(X, W, targets, d_logprob, d_lse):
    """(dX, dW, dl)."""
    p = linear_logprobs(X, W, targets)[2]
    g = np.where(np.asarray(targets) >= 0, d_logprob, 0.0)
    dl = (d_lse - g)[:, None] * p
    for t, v in enumerate(targets):
        if v >= len(W):
            dl[t] = np.nan if g[t] != 0 or d_lse[t] != 0 else 0.0
        elif v >= 0:
            dl[t, v] += g[t]
    return dl @ W, dl.T @ X, dl


# ---- AdamW ----

BLOCK = 128


def offsets(numels):
    """Where each tensor's state begins, and the state's length."""
    at, n = [], 0
    for k in numels:
        at.append(n)
        n += -(-k // BLOCK) * BLOCK
    return at, n


def mix(x):
    """32 bits of noise from 32 (an array of uint64 below 2^32)."""
    x = np.asarray(x, dtype=np.uint64)
    x = x ^ (x >> np.uint64(16))
    x = x * np.uint64(0x9E3779B9) & np.uint64(0xFFFFFFFF)
    x = x ^ (x >> np.uint64(15))
    x = x * np.uint64(0xBB67AE85) & np.uint64(0xFFFFFFFF)
    return x ^ (x >> np.uint64(16))


def noise(i, seed, step):
    """(16 bits for m, 16 for sqrt(v)) of the places i in the state."""
    low = (1 << 32) - 1
    key = int(mix((int(mix((int(mix(seed & low)) + (seed >> 32)) & low)) + step) & low))
    i = np.asarray(i, dtype=np.uint64)
    base = np.uint64(key) ^ mix(i >> np.uint64(32))
    r = mix((i + base) & np.uint64(low))
    return r & np.uint64(0xFFFF), r >> np.uint64(16)


def e4m3(code):
    """The value of e4m3 codes: a sign, four bits of exponent (bias 7), three of fraction."""
    code = np.asarray(code).astype(np.int64)
    e, f = code >> 3 & 15, code & 7
    x = np.where(e == 0, f * 2.0 ** -9, (8 + f) * 2.0 ** (e - 10.0))
    return np.where(code & 0x7F == 0x7F, np.nan, np.where(code & 0x80, -x, x))


def decode(code, exponent):
    """fp32 values of whole blocks of codes."""
    by = np.repeat(np.asarray(exponent).astype(np.int64) - 134, BLOCK)
    with np.errstate(over="ignore"):
        return np.ldexp(e4m3(code), by).astype(F)


def encode(x, noise16, positive):
    """(codes, exponents) of whole blocks of fp32 values."""
    x = np.asarray(x, dtype=F).reshape(-1, BLOCK)
    codes = np.zeros(x.shape, dtype=np.uint8)
    exps = np.zeros(len(x), dtype=np.uint8)
    noise16 = np.asarray(noise16).reshape(x.shape)
    for b, (row, dither) in enumerate(zip(x, noise16)):
        if not np.all(np.isfinite(row)):
            codes[b], exps[b] = 0x7F, 255
            continue
        most = float(np.abs(row).max())
        field = max(1, int(np.frexp(most)[1]) + 126) if most else 1   # 2^(field - 127) <= most
        exps[b] = field
        s = np.ldexp(np.abs(row).astype(np.float64), 134 - field)     # most in 2^7..2^8
        # its binade, or e4m3's least
        e = np.where(s == 0, -6, np.maximum(np.frexp(s)[1] - 1, -6))
        units = np.ldexp(s, 3 - e)                                    # of a code in that binade
        # 20 bits below a unit, to nearest where fp32 holds no more
        units = (np.rint(units * 2.0 ** 20) + dither.astype(np.float64) * 16.0) // 2.0 ** 20
        code = np.where(e == -6, 0, (e + 6) * 8).astype(np.int64) + units.astype(np.int64)
        if positive:
            code = np.where((row > 0) & (code == 0), 1, code)
        codes[b] = np.where(row < 0, code | 0x80, code).astype(np.uint8)
    return codes.reshape(-1), exps


def moments(g, m, v, beta1, beta2):
    """(m, v, sqrt(v)) after the step, each product and sum rounded to fp32."""
    g, m, v = (np.asarray(a, dtype=F) for a in (g, m, v))
    with np.errstate(over="ignore", invalid="ignore"):
        m = F(beta1) * m + F(1.0 - beta1) * g
        v = F(beta2) * v + F(1.0 - beta2) * g * g
        return m, v, np.sqrt(v)


def adamw(p, m, v, step, lr, beta1, beta2, eps, weight_decay):
    """Parameters after the step in 64 bits, from the moments after it."""
    p, m, v = (np.asarray(a, dtype=np.float64) for a in (p, m, v))
    m, v = m / (1 - beta1 ** step), v / (1 - beta2 ** step)
    return p - lr * (weight_decay * p + m / (np.sqrt(v) + eps))
