"""Plain CPU oracle of the token embedding, the 8-bit moments of AdamW and the gradient norm (float64).

TEST INFRASTRUCTURE ONLY: the product path never calls it and shares no code with it. AdamW itself is
``adamw_oracle.adamw_step``.

  out[n] = scale W[id_n]                                   (0 where W does not hold the id)
  dW[v]  = scale sum_{n: id_n = v, id_n != padding} dOut[n]
  norm   = sqrt(sum g^2),  factor = min(1, max_norm / (norm + 1e-6))

8-bit moments: blocks of 32 elements in units U = 2^(s - 127). A code c with k mantissa bits stands for
q(c) U, q(c) = c below 2^k, else (2^k + c mod 2^k) 2^(c // 2^k - 1). s puts the block's largest magnitude a
into the topmost binade of codes, [2^(14+k), 2^(15+k)) units, or one binade below it where a / 2^floor(log2 a)
>= 2 - 2^-k (it could round past the last code there), and s >= 1. A value between two codes takes the upper one
where the place between them plus u reaches 1, u = 16 bits of a hash / 2^16.
"""
from __future__ import annotations

import numpy as np

BLOCK = 32


def embedding(w, ids, scale=1.0, v_begin=0):
    ids = np.asarray(ids, dtype=np.int64) - v_begin
    held = (ids >= 0) & (ids < w.shape[0])
    out = np.zeros((ids.size, w.shape[1]))
    out[held] = scale * w[ids[held]].astype(np.float64)
    return out


def embedding_grad(ids, dout, v, scale=1.0, padding=None, v_begin=0):
    """(dW, number of tokens per id, sum of |scale dOut| per element): the latter two bound rounding errors."""
    dw, mag, count = np.zeros((v, dout.shape[1])), np.zeros((v, dout.shape[1])), np.zeros(v, dtype=np.int64)
    for i, x in zip(np.asarray(ids, dtype=np.int64), dout.astype(np.float64)):
        r = i - v_begin
        if 0 <= r < v and i != padding:
            dw[r] += scale * x
            mag[r] += np.abs(scale * x)
            count[r] += 1
    return dw, count, mag


def norm(tensors, max_norm=np.inf):
    n = np.sqrt(sum(float(np.sum(np.asarray(t, dtype=np.float64) ** 2)) for t in tensors))
    return n, min(1.0, max_norm / (n + 1e-6))


def pair_uniform(place, n, seed):
    """u of elements place .. place + n - 1 (place even)."""
    m = 0xFFFFFFFF
    out = np.empty(n, dtype=np.float64)
    for i in range(n):
        x = (((place + i) // 2) * 0x9E3779B9 + seed) & m
        x = ((x ^ (x >> 16)) * 0x6A09E667) & m
        x = ((x ^ (x >> 15)) * 0xBB67AE85) & m
        x ^= x >> 16
        out[i] = (x >> 16 if (place + i) % 2 else x & 0xFFFF) / 65536.0
    return out


def units(x, k):
    """Unit byte of each block of x (float64, finite)."""
    out = []
    for i in range(0, x.size, BLOCK):
        a = float(np.max(np.abs(x[i:i + BLOCK])))
        if a == 0:
            out.append(1)
            continue
        f, e = np.frexp(a)                       # a = f 2^e, 1/2 <= f < 1
        e = int(e) - 1 + (1 if 2 * f >= 2 - 2.0 ** -k else 0)
        out.append(max(1, e + 127 - (14 + k)))
    return np.array(out, dtype=np.int64)


def place_between(x, s, k):
    """(code of the place x holds, as a real number: integer part the code below; size of a code there) of
    magnitudes x with unit bytes s per element."""
    y = np.abs(x) / np.ldexp(1.0, s - 127)
    h = np.maximum(np.frexp(y)[1] - 1 - k, 0)
    return y / np.ldexp(1.0, h) + h * 2.0 ** k, np.ldexp(1.0, s - 127 + h)


def value(codes, s, k):
    """What codes (magnitudes) stand for, s the unit byte per element."""
    c = np.asarray(codes, dtype=np.int64)
    h, f = c >> k, c & (2 ** k - 1)
    return np.where(h == 0, f, (2 ** k + f) * 2.0 ** (np.maximum(h, 1) - 1)) * np.ldexp(1.0, s - 127)
