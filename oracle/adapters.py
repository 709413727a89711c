"""Float64 oracle of the adapters, the dropout and the token loss -- test infrastructure, not part of the product.

Plain numpy from the definitions, one adapter and one token at a time.  Arrays are on the host; float64 in, float64
out.  Each product also has its `*_abs` bound: the sum of the absolute values of its terms, which the rounding error
of any order of summation is a multiple of.
"""
from __future__ import annotations

import numpy as np

_W = 0xFFFFFFFF


def philox4x32(counter, key, rounds: int):
    """Philox4x32 (Salmon et al., SC'11, Sec. 3.3) of 4 counter words under 2 key words, Python integers."""
    c, k = list(counter), list(key)
    for _ in range(rounds):
        p0, p1 = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(p1 >> 32) ^ c[1] ^ k[0], p1 & _W, (p0 >> 32) ^ c[3] ^ k[1], p0 & _W]
        k = [(k[0] + 0x9E3779B9) & _W, (k[1] + 0xBB67AE85) & _W]
    return c


def drop_factor(rows: int, cols: int, p: float, seed: int, offset: int) -> np.ndarray:
    """0 where an element is dropped, 1 / (1 - round(65536 p) / 65536) where it is kept."""
    if p == 0.0:
        return np.ones((rows, cols))
    thr = int(round(p * 65536))
    key = (seed & _W, seed >> 32 & _W)
    f = np.zeros((rows, cols))
    for t in range(rows):
        for c in range((cols + 7) // 8):
            w = philox4x32((c, t, offset & _W, offset >> 32 & _W), key, 7)
            for e in range(min(8, cols - 8 * c)):
                if (w[e // 2] >> (16 * (e % 2)) & 0xFFFF) >= thr:
                    f[t, 8 * c + e] = 65536.0 / (65536 - thr)
    return f


def dropout(x, residual, p, seed, offset):
    f = drop_factor(*x.shape, p, seed, offset)
    out = np.where(f > 0, np.where(f > 0, x, 0.0) * f, 0.0)
    return out if residual is None else residual + out


def _scale(scale, a):
    return 1.0 if scale is None else float(scale[a])


def adapter_forward(x, a, b, ids, base=None, scale=None, f=None):
    """(y, u, |y| bound, |u| bound) with x [R, n_in], a [n, r, n_in], b [n, r, n_out], ids [R] (anything outside
    0 .. n - 1: no adapter), f the drop factors of x or None."""
    rows, n, rank = len(ids), a.shape[0], a.shape[1]
    y = np.zeros((rows, b.shape[2])) if base is None else base.copy()
    ya = np.abs(y)
    u, ua = np.zeros((rows, rank)), np.zeros((rows, rank))
    for t in range(rows):
        if not 0 <= ids[t] < n:
            continue
        xt = x[t] if f is None else np.where(f[t] > 0, x[t], 0.0) * f[t]
        A, B, s = a[ids[t]], b[ids[t]], _scale(scale, ids[t])
        u[t], ua[t] = A @ xt, np.abs(A) @ np.abs(xt)
        y[t] += s * (B.T @ u[t])
        ya[t] += abs(s) * (np.abs(B).T @ ua[t])
    return y, u, ya, ua


def adapter_backward(x, dy, a, b, ids, u, base=None, scale=None, f=None):
    """(dA, dB, dx) and their bounds."""
    rows, n = len(ids), a.shape[0]
    da, db = np.zeros_like(a), np.zeros_like(b)
    daa, dba = np.zeros_like(a), np.zeros_like(b)
    dx = np.zeros((rows, a.shape[2])) if base is None else base.copy()
    dxa = np.abs(dx)
    for t in range(rows):
        i = ids[t]
        if not 0 <= i < n:
            continue
        s = _scale(scale, i)
        ft = np.ones(a.shape[2]) if f is None else f[t]
        xt = np.where(ft > 0, x[t], 0.0) * ft
        du, dua = s * (b[i] @ dy[t]), abs(s) * (np.abs(b[i]) @ np.abs(dy[t]))
        da[i] += np.outer(du, xt)
        daa[i] += np.outer(dua, np.abs(xt))
        db[i] += s * np.outer(u[t], dy[t])
        dba[i] += abs(s) * np.outer(np.abs(u[t]), np.abs(dy[t]))
        dx[t] += ft * (a[i].T @ du)
        dxa[t] += ft * (np.abs(a[i]).T @ dua)
    return (da, db, dx), (daa, dba, dxa)


def token_loss(z, target, weight=None):
    """(loss [R], gradient [R, V]); masked: target outside the vocabulary or weight 0."""
    rows, vocab = z.shape
    loss, grad = np.zeros(rows), np.zeros((rows, vocab))
    for t in range(rows):
        w = 1.0 if weight is None else float(weight[t])
        if not 0 <= target[t] < vocab or w == 0.0:
            continue
        top = z[t].max()
        if top == -np.inf:      # nothing is possible
            loss[t] = np.inf
            continue
        e = np.exp(z[t] - top)
        loss[t] = w * (np.log(e.sum()) + (top - z[t, target[t]]))
        grad[t] = w * e / e.sum()
        grad[t, target[t]] -= w
    return loss, grad
