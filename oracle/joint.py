"""Oracle of the joint-latent cache (float64 numpy, plain loops): its pages,
what an append leaves in them, attention over its tokens in either form."""

from __future__ import annotations

import math

import numpy as np

from .serving import PAGE


def place(rank, rope_dim, cache, s, j):
    """Element (bf16) or byte (e4m3) of column j of slot s in a page: 16-byte
    pieces change places by the slot."""
    width = rank + rope_dim
    per = 8 if cache == "bf16" else 16
    g = math.gcd(width // per, 16)
    return s * width + ((j // per) ^ (s // (16 // g)) % g) * per + j % per


def page_elems(rank, rope_dim, cache):
    return PAGE * (rank + rope_dim + (2 if cache == "e4m3" else 0))


def e4m3_value(byte):
    """The value of an e4m3 byte (sign, 4 exponent bits of bias 7, 3 mantissa bits)."""
    byte = np.asarray(byte, np.int64)
    sign, e, m = np.where(byte >= 128, -1.0, 1.0), byte // 8 % 16, byte % 8
    x = np.where(e == 0, m / 8.0 * 2.0 ** -6, (1 + m / 8.0) * 2.0 ** (e - 7.0))
    return np.where(byte % 128 == 127, np.nan, sign * x)


def quantized(x):
    """x [n, w] to the nearest e4m3 numbers under each row's least power of two
    2^e, -112 <= e <= 119, with max|x| <= 448 2^e; and e [n]."""
    e = np.array([next((k for k in range(-112, 119) if np.max(np.abs(row), initial=0.0) <= 448.0 * 2.0 ** k), 119)
                  for row in x])
    y = np.clip(x / 2.0 ** e[:, None], -448.0, 448.0)
    step = 2.0 ** (np.maximum(np.floor(np.log2(np.abs(y) + 1e-300)), -6.0) - 3.0)
    return np.rint(y / step) * step, e          # rint: half to even


def tokens(pool, ids, n, rank, rope_dim, cache, raw=None):
    """Latents [n, rank] and keys [n, rope_dim] of the first n slots of pages `ids`
    of a pool [pages, page_elems] of float64 values (bf16) or bytes (e4m3)."""
    j = np.arange(rank + rope_dim)
    x = np.zeros((n, rank + rope_dim))
    for t in range(n):
        page, s = pool[ids[t // PAGE]], t % PAGE
        row = page[place(rank, rope_dim, cache, s, j)]
        if cache == "e4m3":
            row = e4m3_value(row)
            row[:rank] *= 2.0 ** (float(page[PAGE * (rank + rope_dim) + s]) - 127)
            row[rank:] *= 2.0 ** (float(page[PAGE * (rank + rope_dim + 1) + s]) - 127)
        x[t] = row
    return x[:, :rank], x[:, rank:]


def attend(q, c, k, W_keys, W_values, seen, scale):
    """q [rows, H, d + p], row i over the first seen[i] of the tokens c [n, r], k
    [n, p]; factors [H, d, r]; the result [rows, H, d]."""
    rows, H, _ = q.shape
    d = W_keys.shape[1]
    out = np.zeros((rows, H, d))
    for h in range(H):
        keys = np.concatenate([c @ W_keys[h].T, k], 1)
        values = c @ W_values[h].T
        for i in range(rows):
            n = seen[i]
            if n < 1:
                continue
            s = keys[:n] @ q[i, h] * scale
            w = np.exp(s - s.max())
            out[i, h] = w @ values[:n] / w.sum()
    return out
