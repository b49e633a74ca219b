"""Attention over a cache in pages, the plain definition (fp64, CPU), one query row at a time.

TEST INFRASTRUCTURE ONLY, like the rest of this package.

Row t of sequence b (its new tokens are rows first[b] .. first[b + 1] - 1) is at position i = len[b] - first[b + 1] + t and attends to
S_i = { j <= i : i - j < l or (i - j) mod l == 0 } among the positions whose page exists, with scores q . k / sqrt(d); query head h reads key
head h // (heads // kv_heads).  Position p is in slot p % page_size of page table[b, p // page_size].

Pins (tests/test_oracle_rotation.py): equal to oracle.attention for whole sequences in shuffled pages, whatever the rest of the pages holds.
"""
from __future__ import annotations

import numpy as np


def positions(first, length):
    """(sequence, position) of every row that belongs to one; sequence -1 for the rest."""
    seq, pos = np.full(max(int(first[-1]), 0), -1), np.zeros(max(int(first[-1]), 0), dtype=np.int64)
    for b in range(len(length)):
        for t in range(first[b], first[b + 1]):
            seq[t], pos[t] = b, length[b] - first[b + 1] + t
    return seq, pos


def slots(table_row, page_size: int, num_pages: int, p):
    """(page, slot) of positions p, page -1 where there is none."""
    p = np.asarray(p)
    which = p // page_size
    inside = which < len(table_row)
    page = np.where(inside, np.asarray(table_row)[np.minimum(which, max(len(table_row) - 1, 0))] if len(table_row) else -1, -1)
    return np.where((page >= 0) & (page < num_pages), page, -1), p % page_size


def attended(i: int, stride: int):
    j = np.arange(i + 1)
    return j[(i - j < stride) | ((i - j) % stride == 0)]


def paged_attention(Q, K, V, first, length, table, stride: int):
    """Q [rows, heads, d]; K, V [pages, page_size, kv_heads, d].  Returns (out [rows, heads, d], lse [heads, rows], weight [rows, heads, d])
    for the rows of the sequences, NaN for the others; `weight` is sum_j softmax_j |v_j|, what the weights' rounding is measured by.  A row
    without keys: zeros and -inf."""
    Q = np.asarray(Q, dtype=np.float64)
    rows, heads, d = Q.shape
    pages, page_size, kv, _ = K.shape
    out, lse, weight = np.full(Q.shape, np.nan), np.full((heads, rows), np.nan), np.full(Q.shape, np.nan)
    seq, pos = positions(first, length)
    for t in range(len(seq)):
        if seq[t] < 0:
            continue
        out[t], lse[:, t], weight[t] = 0.0, -np.inf, 0.0
        if pos[t] < 0:
            continue
        page, slot = slots(table[seq[t]], page_size, pages, attended(int(pos[t]), stride))
        page, slot = page[page >= 0], slot[page >= 0]
        if len(page) == 0:
            continue
        k, v = K[page, slot].astype(np.float64), V[page, slot].astype(np.float64)     # [keys, kv, d]
        for h in range(heads):
            g = h // (heads // kv)
            s = k[:, g] @ Q[t, h] / np.sqrt(float(d))
            top = s.max()
            e = np.exp(s - top)
            z = e.sum()
            lse[h, t] = top + np.log(z)
            out[t, h] = e @ v[:, g] / z
            weight[t, h] = e @ np.abs(v[:, g]) / z
    return out, lse, weight
