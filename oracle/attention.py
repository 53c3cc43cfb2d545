"""CPU oracle of the paged cache and its attention (numpy, float64).

TEST INFRASTRUCTURE ONLY: imported by ``tests/``; the product never imports it and it shares no code with the HIP path.

Token by token from the definitions: position ``p = kv_len - n_new + i`` of new token ``i`` lies in slot ``p % page_size`` of the
page that entry ``p // page_size`` of the sequence's table names; an entry that names none holds nothing.  A pair (a, b) of channels
turns to ``(a c - b s, a s + b c)``.  In 4 bits a group of 64 channels becomes ``lo`` and ``step`` and whole numbers 0 .. 15.
Attention: ``sum_j e^{x_j} v_j / sum_j e^{x_j}`` over the keys that a token sees, 0 where it sees none.
"""
from __future__ import annotations

import numpy as np


def new_tokens(first, kv_len, n_tokens):
    """Of every new token (sequence, position); the sequence is -1 where no sequence has it."""
    where = np.full((n_tokens, 2), -1, dtype=np.int64)
    for s, held in enumerate(kv_len):
        lo, hi = int(first[s]), int(first[s + 1])
        for i in range(hi - lo):
            where[lo + i] = s, int(held) - (hi - lo) + i
    return where


def place(table_row, p, page_size, n_pages, max_kv):
    """(page, slot) of a position, or None."""
    if p < 0 or p >= max_kv or p // page_size >= len(table_row):
        return None
    page = int(table_row[p // page_size])
    return (page, p % page_size) if 0 <= page < n_pages else None


def turned(rows, turn, rot, neighbours):
    """Rows [..][channel] with the first ``rot`` channels turned by ``turn`` [rot / 2][2]."""
    out = np.array(rows, dtype=np.float64)
    for i in range(rot // 2):
        a, b = (2 * i, 2 * i + 1) if neighbours else (i, i + rot // 2)
        c, s = float(turn[i, 0]), float(turn[i, 1])
        x, y = out[..., a].copy(), out[..., b].copy()
        out[..., a], out[..., b] = x * c - y * s, x * s + y * c
    return out


def attention(q, keys, values, pos, there, scale, window, sinks):
    """One query row against a sequence: keys, values [n][channel], ``there`` [n] truth values.  Returns the row, the same sum of
    absolute values (what relative errors of weights and values are relative to), and how many keys were seen."""
    n = len(keys)
    j = np.arange(n)
    sees = there & (j <= pos)
    if window:
        sees &= (j > pos - window) | (j < sinks)
    if not sees.any():
        return np.zeros(values.shape[1]), np.zeros(values.shape[1]), 0
    x = scale * (keys[sees] @ q)
    top = x.max()
    w = np.exp(x - (top if top > -np.inf else 0.0))
    total = w.sum()
    if total == 0.0:
        return np.zeros(values.shape[1]), np.zeros(values.shape[1]), int(sees.sum())
    return (w @ values[sees]) / total, (w @ np.abs(values[sees])) / total, int(sees.sum())
