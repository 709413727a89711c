"""Float64 oracle of the layer norm, the preference loss and the AdamW step -- test infrastructure, not part of the product.

Plain numpy from the definitions, one row, one token and one block at a time.  Arrays are on the host; float64 in,
float64 out.
"""
from __future__ import annotations

import numpy as np

from .adapters import philox4x32

_W = 0xFFFFFFFF


# -------------------------------------------------------------- layer norm --
def norm_forward(h, gain=None, bias=None, eps=1e-5, rms=False, mask=None):
    """(y, mean, rstd) of the rows of h; zeros for rows whose mask is 0."""
    rows, cols = h.shape
    y, mean, rstd = np.zeros((rows, cols)), np.zeros(rows), np.zeros(rows)
    for t in range(rows):
        if mask is not None and not mask[t]:
            continue
        if not rms:
            mean[t] = np.sum(h[t]) / cols
        rstd[t] = 1.0 / np.sqrt(np.sum((h[t] - mean[t]) ** 2) / cols + eps)
        y[t] = (h[t] - mean[t]) * rstd[t]
        if gain is not None:
            y[t] = y[t] * gain
        if bias is not None:
            y[t] = y[t] + bias
    return y, mean, rstd


def norm_backward(h, dy, mean, rstd, gain=None, rms=False, mask=None, base=None):
    """(dx, dgain, dbias) for statistics as given (zeros for the mean of an rms norm)."""
    rows, cols = h.shape
    dx = np.zeros((rows, cols)) if base is None else base.copy()
    dgain, dbias = np.zeros(cols), np.zeros(cols)
    for t in range(rows):
        if mask is not None and not mask[t]:
            continue
        xh = (h[t] - (0.0 if rms else mean[t])) * rstd[t]
        c = dy[t] if gain is None else dy[t] * gain
        back = c - xh * (np.sum(c * xh) / cols)
        if not rms:
            back = back - np.sum(c) / cols
        dx[t] += rstd[t] * back
        dgain += dy[t] * xh
        dbias += dy[t]
    return dx, dgain, dbias


# --------------------------------------------------------- preference loss --
def token_logp(z, target):
    """(log probability of the target, probabilities) of one token's logits; a token without a finite logit has none."""
    top = np.max(z)
    if top == -np.inf:
        return -np.inf, None
    e = np.exp(z - top)
    total = np.sum(e)
    return z[target] - top - np.log(total), e / total


def softplus(x):
    return np.logaddexp(0.0, x)


def preference_loss(z, target, offsets, ref=None, weight=None, beta=0.1, smoothing=0.0):
    """(loss [n], logp [2 n], dz [rows, vocab])."""
    rows, vocab = z.shape
    n = len(offsets) // 2
    logp, loss, dz = np.zeros(2 * n), np.zeros(n), np.zeros((rows, vocab))
    probs = {}
    for s in range(2 * n):
        for t in range(offsets[s], offsets[s + 1]):
            if 0 <= target[t] < vocab:
                lp, probs[t] = token_logp(z[t], target[t])
                logp[s] += lp
    for i in range(n):
        w = 1.0 if weight is None else float(weight[i])
        if w == 0.0:
            continue
        ratio = [logp[s] - (0.0 if ref is None else ref[s]) for s in (2 * i, 2 * i + 1)]
        d = beta * (ratio[0] - ratio[1])
        loss[i] = w * ((1 - smoothing) * softplus(-d) + (smoothing * softplus(d) if smoothing else 0.0))
        slope = w * beta * (smoothing - 1.0 / (1.0 + np.exp(d)))
        for s, sign in ((2 * i, 1.0), (2 * i + 1, -1.0)):
            for t in range(offsets[s], offsets[s + 1]):
                if probs.get(t) is not None:
                    dz[t] = -sign * slope * probs[t]
                    dz[t, target[t]] += sign * slope
    return loss, logp, dz


# -------------------------------------------------------------------- AdamW --
# an 8-bit type: mantissa bits, smallest exponent, exponent of the largest value (1.75 times that power of two)
E4M3 = (3, -6, 8)
E5M2 = (2, -14, 15)
BLOCK = 256


def values_of(kind):
    """The magnitudes that the type's finite codes stand for, in order."""
    bits, low, high = kind
    steps = [n * 2.0 ** (low - bits) for n in range(2 ** bits)]
    for e in range(low, high + 1):
        steps += [(2 ** bits + n) * 2.0 ** (e - bits) for n in range(2 ** bits)]
    return np.array([v for v in steps if v <= 1.75 * 2.0 ** high])


def block_scale(x, kind):
    """The smallest 2^k, k >= -126, that brings the largest magnitude to the type's largest value or below."""
    top = np.max(np.abs(x[np.abs(x) < 2.0 ** 128]), initial=0.0)
    if top == 0.0:
        return 1.0
    k = -126
    while top / 2.0 ** k > 1.75 * 2.0 ** kind[2]:
        k += 1
    return 2.0 ** k


def round_at_random(x, scale, kind, draw, never_zero):
    """The value (times the scale) that each element takes, draw: 16 bits each."""
    grid = values_of(kind)
    out = np.empty_like(x)
    for i, v in enumerate(x):
        if not abs(v) < 2.0 ** 128:
            out[i] = np.nan if kind is E4M3 or np.isnan(v) else np.inf
            continue
        a = abs(v) / scale
        j = int(np.searchsorted(grid, a, side="right")) - 1
        if j + 1 < len(grid) and (a - grid[j]) / (grid[j + 1] - grid[j]) * 65536 > draw[i]:
            j += 1
        if never_zero and a > 0:
            j = max(j, 1)
        out[i] = np.copysign(grid[j] * scale, v)
    return out


def adamw_draws(count, part, tensor, step, seed):
    """16 bits for m and 16 for v of each of a slice's elements."""
    words = [w for q in range(-(-count // 4))
             for w in philox4x32((q, part, tensor, step & _W), (seed & _W, seed >> 32 & _W), 7)]
    words = np.array(words[:count], dtype=np.uint64)
    return (words & np.uint64(0xFFFF)).astype(np.int64), (words >> np.uint64(16)).astype(np.int64)


def adamw_step(tensors, n_groups, step, lr, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, max_norm=0.0, lr_scale=None,
               with_norms=False, seed=0):
    """tensors: dicts of param, grad, m, v [slices, slice] float64 (the values that the states stand for), first_group,
    decay, bits.  Returns (the tensors after the step, with m_scale and v_scale [slices, blocks] for 8-bit states,
    norms)."""
    t = step + 1
    square = np.zeros(n_groups)
    for x in tensors:
        for s in range(x["param"].shape[0]):
            square[x["first_group"] + s] += np.sum(x["grad"][s] ** 2)
    norms = np.sqrt(square)
    out = []
    for index, x in enumerate(tensors):
        y = {k: np.array(x[k], dtype=np.float64) for k in ("param", "m", "v")}
        slices, n = x["param"].shape
        blocks = -(-n // BLOCK)
        if x["bits"] == 8:
            y["m_scale"], y["v_scale"] = (np.array(x[k], dtype=np.float64).reshape(slices, blocks) for k in ("m_scale", "v_scale"))
        for s in range(slices):
            g = x["first_group"] + s
            if (max_norm > 0 or with_norms) and not np.isfinite(norms[g]):
                continue
            c = max_norm / norms[g] if 0 < max_norm < norms[g] else 1.0
            grad = x["grad"][s] * c
            m = beta1 * x["m"][s] + (1 - beta1) * grad
            v = beta2 * x["v"][s] + (1 - beta2) * grad ** 2
            rate = lr if lr_scale is None else lr * float(lr_scale[g])
            p = x["param"][s] * (1 - (rate * weight_decay if x["decay"] else 0.0))
            y["param"][s] = p - rate * (m / (1 - beta1 ** t)) / (np.sqrt(v / (1 - beta2 ** t)) + eps)
            if x["bits"] == 8:
                for_m, for_v = adamw_draws(n, s, index, t, seed)
                for b in range(blocks):
                    i = slice(BLOCK * b, min(n, BLOCK * (b + 1)))
                    y["m_scale"][s, b], y["v_scale"][s, b] = block_scale(m[i], E4M3), block_scale(v[i], E5M2)
                    m[i] = round_at_random(m[i], y["m_scale"][s, b], E4M3, for_m[i], False)
                    v[i] = round_at_random(v[i], y["v_scale"][s, b], E5M2, for_v[i], True)
            y["m"][s], y["v"][s] = m, v
        out.append(y)
    return out, norms
