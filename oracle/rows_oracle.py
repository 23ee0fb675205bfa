"""Plain 64-bit oracle for the operators on rows of a network over tokens (TEST
INFRASTRUCTURE ONLY; shares no code with the HIP path and imports nothing from it).

Matrices are numpy arrays of any float type; everything is computed in float64 from their
values.  A mask is (p, seed, number), p as the caller's binary32 number.
"""

from __future__ import annotations

import numpy as np


def philox4x32(counter, key, rounds=10):
    """Philox4x32 (Salmon, Moraes, Dror, Shaw: "Parallel random numbers: as easy as 1, 2, 3",
    SC 2011, section 4): counter of four and key of two 32-bit numbers, as Python integers (or
    the counter as uint64 arrays: the products fit)."""
    low = 0xFFFFFFFF
    x0, x1, x2, x3 = counter
    k0, k1 = key
    for r in range(rounds):
        if r:
            k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
        p0, p1 = 0xD2511F53 * x0, 0xCD9E8D57 * x2
        x0, x1, x2, x3 = (p1 >> 32) ^ x1 ^ k0, p1 & low, (p0 >> 32) ^ x3 ^ k1, p0 & low
    return x0, x1, x2, x3


def drop_below(p):
    """round(65536 p) of the binary32 number p, ties to even."""
    return int(np.rint(float(np.float32(p)) * 65536.0))


def kept(n, d, drop):
    """Boolean n x d: the elements that the mask keeps."""
    p, seed, number = drop
    below = drop_below(p)
    i, q = np.meshgrid(np.arange(n, dtype=np.uint64), np.arange(-(-d // 8), dtype=np.uint64),
                       indexing="ij")
    number = np.full(q.shape, number, np.uint64)
    words = philox4x32((q, i, number & np.uint64(0xFFFFFFFF), number >> np.uint64(32)),
                       (seed & 0xFFFFFFFF, seed >> 32))
    out = np.empty((n, -(-d // 8) * 8), bool)
    for j in range(8):
        out[:, j::8] = (words[j // 2] >> np.uint64(16 * (j % 2)) & np.uint64(0xFFFF)) >= below
    return out[:, :d]


def dropout(X, drop):
    """Kept elements times 65536 / (65536 - round(65536 p)), the others 0."""
    X = np.asarray(X, np.float64)
    below = drop_below(drop[0])
    if below == 65536:
        return np.zeros(X.shape)
    return np.where(kept(*X.shape, drop), X * (65536.0 / (65536 - below)), 0.0)


def _maybe(X, drop):
    return np.asarray(X, np.float64) if drop is None else dropout(X, drop)


def embed(ids, E, scale=1.0, drop=None):
    E = np.asarray(E, np.float64)
    out = np.zeros((len(ids), E.shape[1]))
    for t, v in enumerate(ids):
        if 0 <= v < len(E):
            out[t] = scale * E[v]
    return _maybe(out, drop)


def embed_grad(ids, G, n_vocab, scale=1.0, drop=None):
    """(gradient, sum of the absolute values of the terms of each of its entries, terms of
    each row)."""
    G = _maybe(G, drop)
    dE, S = np.zeros((n_vocab, G.shape[1])), np.zeros((n_vocab, G.shape[1]))
    count = np.zeros(n_vocab, np.int64)
    for t, v in enumerate(ids):
        if 0 <= v < n_vocab:
            dE[v] += scale * G[t]
            S[v] += np.abs(scale * G[t])
            count[v] += 1
    return dE, S, count


def rmsnorm(X, R=None, w=None, eps=1e-5, drop=None):
    """(h, y)."""
    h = _maybe(X, drop)
    if R is not None:
        h = h + np.asarray(R, np.float64)
    y = h / np.sqrt(np.mean(h * h, axis=1, keepdims=True) + eps)
    return h, y if w is None else y * np.asarray(w, np.float64)


def rmsnorm_grad(H, dY, w=None, eps=1e-5, dR=None, drop=None):
    """(dH, dX, dw), the chain rule written out for one row at a time: y_j = w_j h_j r with
    dr / dh_k = -r^3 h_k / d."""
    H, dY = np.asarray(H, np.float64), np.asarray(dY, np.float64)
    n, d = H.shape
    w = np.ones(d) if w is None else np.asarray(w, np.float64)
    dH, dw = np.zeros((n, d)), np.zeros(d)
    for i in range(n):
        h, g = H[i], dY[i] * w
        r = (np.dot(h, h) / d + eps) ** -0.5
        dr = np.dot(g, h)                       # d loss / d r
        dH[i] = g * r + dr * (-r ** 3 * h / d)
        dw += dY[i] * h * r
    if dR is not None:
        dH = dH + np.asarray(dR, np.float64)
    return dH, _maybe(dH, drop), dw


def e4m3_values():
    """The 256 numbers of the OCP 8-bit format with 4 exponent bits (bias 7) and 3 mantissa
    bits: no infinities, S.1111.111 is NaN."""
    out = np.empty(256)
    for b in range(256):
        sign, e, m = -1.0 if b & 0x80 else 1.0, b >> 3 & 15, b & 7
        if e == 15 and m == 7:
            out[b] = np.nan
        elif e == 0:
            out[b] = sign * m / 8 * 2.0 ** -6
        else:
            out[b] = sign * (1 + m / 8) * 2.0 ** (e - 7)
    return out


def e4m3_half_step(x):
    """Half the distance between neighbours of the format at magnitude |x|."""
    e = np.floor(np.log2(np.maximum(np.abs(x), 2.0 ** -6)))
    return 2.0 ** (np.minimum(e, 8) - 4)
