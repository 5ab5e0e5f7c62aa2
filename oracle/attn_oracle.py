"""Attention over a paged key-value cache in 64 bits, from its definition (test infrastructure; plain
NumPy loops, no code shared with the library).

Arrays hold the values that the 16-bit inputs stand for, as float64.  Layouts are those of
include/vq.h: K pages [page][kv head][slot][dim], V pages [page][kv head][dim][slot].
"""
from __future__ import annotations

import numpy as np

__all__ = ["cache_of", "attention", "append", "copy_pages"]


def cache_of(k_pages, v_pages, table_row, n):
    """(keys, values) [n, kv heads, dim] of the first n tokens of the sequence whose pages table_row lists."""
    size = k_pages.shape[2]
    k = np.empty((n, k_pages.shape[1], k_pages.shape[3]))
    v = np.empty_like(k)
    for j in range(n):
        page, slot = table_row[j // size], j % size
        k[j] = k_pages[page, :, slot, :]
        v[j] = v_pages[page, :, :, slot]
    return k, v


def attention(q, k_pages, v_pages, table, kv_len, q_start, scale):
    """out [T, heads, dim], lse [T, heads], and for bounds of the rounding: sum p |v| / l, the largest |q|.|k| * scale
    and the number of attended tokens of every row."""
    T, H, D = q.shape
    kv = k_pages.shape[1]
    out, lse, mean_abs = np.zeros((T, H, D)), np.full((T, H), -np.inf), np.zeros((T, H, D))
    logit_abs, count = np.zeros((T, H)), np.zeros((T, H), dtype=np.int64)
    for s in range(len(kv_len)):
        first, last = q_start[s], q_start[s + 1]
        if last == first:
            continue
        k, v = cache_of(k_pages, v_pages, table[s], kv_len[s])
        for t in range(first, last):
            n = kv_len[s] - last + t + 1
            if n <= 0:
                continue
            for h in range(H):
                kh, vh = k[:n, h // (H // kv)], v[:n, h // (H // kv)]
                with np.errstate(invalid="ignore", over="ignore"):
                    x = (kh @ q[t, h]) * scale
                    m = x.max()
                    p = np.exp(x - m)
                    l = p.sum()
                    out[t, h] = (p / l) @ vh
                    lse[t, h] = m + np.log(l)
                    mean_abs[t, h] = (p / l) @ np.abs(vh)
                    logit_abs[t, h] = scale * (np.abs(kh) @ np.abs(q[t, h])).max()
                count[t, h] = n
    return out, lse, mean_abs, logit_abs, count


def append(k, v, k_pages, v_pages, table, kv_len, q_start):
    """The pages with the new tokens in them (copies)."""
    k_pages, v_pages, size = k_pages.copy(), v_pages.copy(), k_pages.shape[2]
    for s in range(len(kv_len)):
        for t in range(q_start[s], q_start[s + 1]):
            pos = kv_len[s] - q_start[s + 1] + t
            if pos < 0 or not 0 <= table[s][pos // size] < len(k_pages):
                continue
            k_pages[table[s][pos // size], :, pos % size, :] = k[t]
            v_pages[table[s][pos // size], :, :, pos % size] = v[t]
    return k_pages, v_pages


def copy_pages(buffers, pairs):
    """The buffers [n_buffers, n_pages, ...] after every pair in turn (a copy)."""
    buffers = buffers.copy()
    for a, b in pairs:
        buffers[:, b] = buffers[:, a]
    return buffers
