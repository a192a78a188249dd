"""CPU oracle of what is tuned around frozen matrices, in binary64: dropout by a counter-based generator, token embeddings and
low-rank adapters, with their gradients.

TEST INFRASTRUCTURE ONLY: tests and the smoke check may import this; the GPU library never does, and this
module imports nothing from the GPU package.
"""
from __future__ import annotations

import numpy as np

LOW = 0xFFFFFFFF


def philox(counter, key, rounds=10):
    """Philox 4x32 on Python's integers: four words and two words in, four words out."""
    c, k = list(counter), list(key)
    for _ in range(rounds):
        a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(b >> 32) ^ c[1] ^ k[0], b & LOW, (a >> 32) ^ c[3] ^ k[1], a & LOW]
        k = [(k[0] + 0x9E3779B9) & LOW, (k[1] + 0xBB67AE85) & LOW]
    return c


def limit(p):
    """p as a multiple of 2^-16, in those units."""
    return int(p * 65536.0 + 0.5)


def keep(seed, p, M, n, call=0):
    """Which elements of [M][n] stay, and the factor of those that do.  seed: (key, number) of 64 bits each."""
    key, number = int(seed[0]) % 2 ** 64, (int(seed[1]) + call) % 2 ** 64
    out = np.empty((M, n), dtype=bool)
    for row in range(M):
        for block in range((n + 7) // 8):
            words = philox((block, row, number & LOW, number >> 32), (key & LOW, key >> 32))
            numbers = [w >> s & 0xFFFF for w in words for s in (0, 16)]
            out[row, 8 * block:8 * block + 8] = [v >= limit(p) for v in numbers][:n - 8 * block]
    return out, (1.0 / (1.0 - limit(p) / 65536.0) if limit(p) < 65536 else 0.0)


def dropout(x, seed, p, call=0):
    x = np.asarray(x, dtype=np.float64)
    stays, factor = keep(seed, p, x.shape[0], x.shape[1], call)
    return np.where(stays, x * factor, 0.0)


def embedding(tokens, table, scale=1.0):
    """Rows of zeros for tokens outside the table."""
    table = np.asarray(table, dtype=np.float64)
    return np.array([scale * table[t] if 0 <= t < len(table) else np.zeros(table.shape[1]) for t in tokens])


def embedding_backward(tokens, dout, vocab, scale=1.0):
    """-> the gradient, and for each row the sum of magnitudes and the number of its terms"""
    dout = np.asarray(dout, dtype=np.float64)
    grad, size, count = np.zeros((vocab, dout.shape[1])), np.zeros((vocab, dout.shape[1])), np.zeros(vocab, dtype=np.int64)
    for t, row in zip(tokens, dout):
        if 0 <= t < vocab:
            grad[t] += scale * row
            size[t] += abs(scale) * np.abs(row)
            count[t] += 1
    return grad, size, count


def adapter_rows(lens, ids, n_adapters):
    """(adapter, first row, row behind the last) of the sequences that have one."""
    first = np.concatenate([[0], np.cumsum(lens)])
    return [(a, f, f + n) for a, f, n in zip(ids, first, lens) if 0 <= a < n_adapters and n]


def adapters(x, a, b, lens, ids, scales, base=None):
    """x: [M][K] (dropped already), a: [n][r][K], b: [n][N][r].  -> y [M][N], h [M][r]"""
    x, a, b = (np.asarray(t, dtype=np.float64) for t in (x, a, b))
    y = np.zeros((len(x), b.shape[1])) if base is None else np.array(base, dtype=np.float64)
    h = np.zeros((len(x), a.shape[1]))
    for i, f, e in adapter_rows(lens, ids, len(a)):
        h[f:e] = x[f:e] @ a[i].T
        y[f:e] += scales[i] * (h[f:e] @ b[i].T)
    return y, h


def adapters_backward(x, dy, h, a, b, lens, ids, scales, stays=1.0):
    """x dropped already; stays: the factors of dropout.  -> dx without its base, da, db"""
    x, dy, h, a, b = (np.asarray(t, dtype=np.float64) for t in (x, dy, h, a, b))
    dx, da, db = np.zeros_like(x), np.zeros_like(a), np.zeros_like(b)
    for i, f, e in adapter_rows(lens, ids, len(a)):
        g = scales[i] * (dy[f:e] @ b[i])
        dx[f:e] = g @ a[i]
        da[i] += g.T @ x[f:e]
        db[i] += scales[i] * (dy[f:e].T @ h[f:e])
    return dx * stays, da, db
