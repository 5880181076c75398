"""Float64 NumPy definitions of the operators on rows and of the relative
position bias, independent of the HIP code: the counter-based dropout mask
(Philox4x32-10, Salmon et al. 2011), layer norm with its backward pass, the
position buckets (compared in integers) and the bias with its gradient."""
from __future__ import annotations

import numpy as np

_M = (0xD2511F53, 0xCD9E8D57)
_W = (0x9E3779B9, 0xBB67AE85)
_LOW = 0xFFFFFFFF


def philox4x32(counter, key, rounds=10):
    """The generator on Python integers: four 32-bit words."""
    c, k = list(counter), list(key)
    for _ in range(rounds):
        p0, p1 = _M[0] * c[0], _M[1] * c[2]
        c = [(p1 >> 32) ^ c[1] ^ k[0], p1 & _LOW, (p0 >> 32) ^ c[3] ^ k[1], p0 & _LOW]
        k = [(k[0] + _W[0]) & _LOW, (k[1] + _W[1]) & _LOW]
    return c


def numbers(seed, n, rows, cols, row0=0):
    """The 16-bit number of every element: [rows][cols]."""
    pieces = (cols + 7) // 8
    low = np.uint64(_LOW)
    c = [np.broadcast_to(np.arange(pieces, dtype=np.uint64), (rows, pieces)),
         np.broadcast_to(np.arange(row0, row0 + rows, dtype=np.uint64)[:, None], (rows, pieces)),
         np.full((rows, pieces), n & _LOW, np.uint64),
         np.full((rows, pieces), (n >> 32) & _LOW, np.uint64)]
    k = [seed & _LOW, (seed >> 32) & _LOW]
    for _ in range(10):
        p0, p1 = np.uint64(_M[0]) * c[0], np.uint64(_M[1]) * c[2]
        c = [(p1 >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), p1 & low,
             (p0 >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), p0 & low]
        k = [(k[0] + _W[0]) & _LOW, (k[1] + _W[1]) & _LOW]
    out = np.empty((rows, pieces, 8), np.int64)
    for u in range(8):
        out[:, :, u] = (c[u // 2] >> np.uint64(16 * (u % 2))) & np.uint64(0xFFFF)
    return out.reshape(rows, pieces * 8)[:, :cols]


def threshold(p):
    return int(np.floor(65536 * p + 0.5))


def mask(p, seed, n, rows, cols, row0=0):
    """(kept, scale): which elements stay, and their factor."""
    t = threshold(p)
    kept = numbers(seed, n, rows, cols, row0) >= t
    return kept, 65536 / (65536 - t) if t < 65536 else 0.0


def dropout(x, kept=None, scale=1.0):
    return x if kept is None else np.where(kept, x * scale, 0.0)


def layer_norm(s, weight, bias, eps):
    """(out, mean, rstd) of rows s."""
    mean = s.mean(1)
    rstd = 1 / np.sqrt(((s - mean[:, None]) ** 2).mean(1) + eps)
    z = (s - mean[:, None]) * rstd[:, None]
    return z * (1 if weight is None else weight) + (0 if bias is None else bias), mean, rstd


def layer_norm_grad(grad, s, weight, mean, rstd):
    """(gradient of s, of the weight, of the bias)."""
    z = (s - mean[:, None]) * rstd[:, None]
    h = grad * (1 if weight is None else weight)
    g = rstd[:, None] * (h - h.mean(1, keepdims=True) - z * (h * z).mean(1, keepdims=True))
    return g, (grad * z).sum(0), grad.sum(0)


def bucket(n, num_buckets, max_distance, bidirectional):
    """Bucket of one distance n = query position - key position, by comparing
    integer powers."""
    side = num_buckets // 2 if bidirectional else num_buckets
    add = 0
    if n < 0:
        if bidirectional:
            add, n = side, -n
        else:
            n = 0
    e = side // 2
    if n < e:
        return add + n
    steps, j = side - e, 0
    while j + 1 < steps and n ** steps >= e ** (steps - j - 1) * max_distance ** (j + 1):
        j += 1
    return add + e + j


def bucket_matrix(first, Q, K, of):
    """Buckets of Q queries from position `first` on and keys 0 .. K-1; `of`
    maps a distance to its bucket."""
    n = (first + np.arange(Q))[:, None] - np.arange(K)[None, :]
    distinct, where = np.unique(n, return_inverse=True)
    return np.array([of(int(v)) for v in distinct])[where].reshape(Q, K)


def position_bias(table, buckets, scores=None):
    """buckets: [B][Q][K]; table: [n][H] -> [B][H][Q][K]."""
    out = np.moveaxis(table[buckets], -1, 1)
    return out if scores is None else out + scores


def position_bias_grad(grad, buckets, num):
    """[num][H] sums of grad [B][H][Q][K] by bucket."""
    out = np.zeros((num, grad.shape[1]))
    for h in range(grad.shape[1]):
        out[:, h] = np.bincount(buckets.reshape(-1), grad[:, h].reshape(-1), num)
    return out
