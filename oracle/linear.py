"""CPU oracle of weights in 4 bits and of log probabilities (numpy, float64).

TEST INFRASTRUCTURE ONLY: imported by ``tests/``; the product never imports it and it shares no code with the HIP path.

Column by column from the definitions: column ``c`` of a row is in word ``c // 128 * 16 + c % 32 // 8 * 4 + c % 128 // 32``, with ``j = c % 8``
from bit ``2 j`` on where j is even and from bit ``2 j + 14`` on where it is odd, and stands for ``lo + step * code`` with the pair
of group ``c // group``.
"""
from __future__ import annotations

import numpy as np


def place(c):
    """(word of the row, first bit) of a column."""
    j = c % 8
    return c // 128 * 16 + c % 32 // 8 * 4 + c % 128 // 32, 2 * j if j % 2 == 0 else 2 * j + 14


def values(words, pairs, group, n_in):
    """What packed rows stand for: words uint32 [n][..], pairs float64 [n][..][2] (step, lo)."""
    out = np.zeros((words.shape[0], n_in))
    for c in range(n_in):
        word, bit = place(c)
        out[:, c] = pairs[:, c // group, 1] + pairs[:, c // group, 0] * (words[:, word] >> np.uint32(bit) & np.uint32(15))
    return out


def packed(x, group, up):
    """Codes [n][n_in] and pairs [n][blocks * 128 / group][2] of rows x (float64); ``up`` rounds a float64 up to the 16-bit type, as a float64."""
    n, n_in = x.shape
    groups = -(-n_in // 128) * (128 // group)
    codes, pairs = np.zeros((n, n_in), np.int64), np.zeros((n, groups, 2))
    for r in range(n):
        for g in range(groups):
            part = x[r, g * group:min(n_in, (g + 1) * group)]
            if len(part) == 0:
                continue
            if not np.isfinite(part).all():
                pairs[r, g] = np.nan
                continue
            lo, hi = part.min(), part.max()
            step = up(np.float64(np.float32(np.float32(hi) - np.float32(lo)) / np.float32(15)))
            pairs[r, g] = step, lo
            if step > 0:                               # the quotient is one of 32 bits: codes next to a border come out the same
                quotient = (part.astype(np.float32) - np.float32(lo)) / np.float32(step)
                codes[r, g * group:g * group + len(part)] = np.clip(np.rint(quotient), 0, 15).astype(np.int64)
    return codes, pairs


def act(g, kind):
    if kind == "silu":
        return g / (1.0 + np.exp(-g))
    return 0.5 * g * (1.0 + np.tanh(np.sqrt(2.0 / np.pi) * (g + 0.044715 * g ** 3)))


def logprobs(x, token, scale, top):
    """Of one row: log p of the token, entropy, alternatives (ids, log p), and the mean of |s - largest|."""
    s = x * scale
    there = np.nonzero(x > -np.inf)[0]
    order = there[np.lexsort((there, -x[there]))][:top]
    ids, tops = np.full(top, -1, np.int64), np.full(top, -np.inf)
    ids[:len(order)] = order
    if len(there) == 0:
        return (-np.inf if 0 <= token < len(x) else 0.0), 0.0, ids, tops, 0.0
    m = s.max()
    e = np.exp(s - m)
    log = np.log(e.sum()) + m
    p = e / e.sum()
    live = p > 0
    tops[:len(order)] = s[order] - log
    return (s[token] - log if 0 <= token < len(x) else 0.0), -(p[live] * (s[live] - log)).sum(), ids, tops, (p[live] * (m - s[live])).sum()
