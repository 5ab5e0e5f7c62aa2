"""Attention over a paged key-value cache in 64 bits, from its definition (test infrastructure; plain
NumPy loops, no code shared with the library).

Arrays hold the values that the 16-bit inputs stand for, as float64.  Layouts are those of
include/vq.h: K pages [page][kv head][slot][dim], V pages [page][kv head][dim][slot].
"""
from __future__ import annotations

import numpy as np

__all__ = ["cache_of", "attention", "append", "copy_pages", "CODE_VALUES", "nearest_code", "scale_for", "append8", "values8"]


def cache_of(k_pages, v_pages, table_row, n):
    """(keys, values) [n, kv heads, dim] of the first n tokens of the sequence whose pages table_row lists."""
    size = k_pages.shape[2]
    k = np.empty((n, k_pages.shape[1], k_pages.shape[3]))
    v = np.empty_like(k)
    for j in range(n):
        page, slot = table_row[j // size], j % size
        if not 0 <= page < len(k_pages):
            k[j] = v[j] = np.nan   # given back: nobody may look there
            continue
        k[j] = k_pages[page, :, slot, :]
        v[j] = v_pages[page, :, :, slot]
    return k, v


def attention(q, k_pages, v_pages, table, kv_len, q_start, scale, window=None, sinks=0):
    """out [T, heads, dim], lse [T, heads], and for bounds of the rounding: sum p |v| / l, the largest |q|.|k| * scale
    and the number of attended tokens of every row.  window: of the tokens up to a row's own the last so many are attended, and the first `sinks`."""
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
            seen = np.arange(n) if window is None else np.array([j for j in range(n) if j > n - 1 - window or j < sinks])
            for h in range(H):
                kh, vh = k[seen, h // (H // kv)], v[seen, h // (H // kv)]
                with np.errstate(invalid="ignore", over="ignore"):
                    x = (kh @ q[t, h]) * scale
                    m = x.max()
                    p = np.exp(x - m)
                    l = p.sum()
                    out[t, h] = (p / l) @ vh
                    lse[t, h] = m + np.log(l)
                    mean_abs[t, h] = (p / l) @ np.abs(vh)
                    logit_abs[t, h] = scale * (np.abs(kh) @ np.abs(q[t, h])).max()
                count[t, h] = len(seen)
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


# ---------------------------------------------------------------------------------------- pages in 8 bits
# The number that a code stands for: sign, 4 bits of exponent (bias 7; 0: subnormal), 3 of fraction; all ones but the sign: no number.
CODE_VALUES = np.array([(-1.0) ** (c >> 7) * (np.nan if c & 127 == 127 else (c & 7) / 8 * 2.0 ** -6 if c >> 3 & 15 == 0
                                               else (1 + (c & 7) / 8) * 2.0 ** ((c >> 3 & 15) - 7)) for c in range(256)])
_MIDDLE = (CODE_VALUES[:126] + CODE_VALUES[1:127]) / 2
LEAST_SCALE = {"f16": 2.0 ** -15, "bf16": 2.0 ** -117}
MOST_VALUE = {"f16": 1.875 * 2.0 ** 15, "bf16": 1.875 * 2.0 ** 127}


def nearest_code(x):
    """Codes of the numbers nearest to x, ties to the even code; NaN for what is no finite number.  |x| is 448 at most."""
    a = np.abs(np.where(np.isfinite(x), x, 0))
    assert (a <= 448).all()
    low, high = np.searchsorted(_MIDDLE, a, side="left"), np.searchsorted(_MIDDLE, a, side="right")   # they differ for a tie
    c = np.where(low % 2 == 0, low, high)
    return np.where(np.isfinite(x), c | np.where(np.signbit(x), 128, 0), 127).astype(np.uint8)


def scale_for(largest, dtype):
    s = LEAST_SCALE[dtype]
    while 448 * s < largest:
        s *= 2
    return s


def append8(k, v, k_codes, k_scales, v_codes, v_scales, table, kv_len, q_start, dtype, max_len=None):
    """(k_codes, k_scales, v_codes, v_scales) with the new tokens in them (copies): codes [page][head][slot][dim] and [page][head][dim][slot],
    scales [page][head][block of 16 slots]."""
    out = [k_codes.copy(), k_scales.copy(), v_codes.copy(), v_scales.copy()]
    size = k_codes.shape[2]
    for x, codes, scales in ((k, out[0], out[1]), (v, out[2].transpose(0, 1, 3, 2), out[3])):
        for s in range(len(kv_len)):
            n = q_start[s + 1] - q_start[s]
            behind = kv_len[s] - q_start[s + 1]
            first, last = max(0, kv_len[s] - n), kv_len[s] if max_len is None else min(kv_len[s], max_len)
            for at in range(first // 16 * 16, last, 16):
                lo, hi = max(at, first), min(at + 16, last)
                page = table[s][at // size]
                if lo >= hi or not 0 <= page < len(codes):
                    continue
                slot, block = at % size, at % size // 16
                for h in range(codes.shape[1]):
                    new = x[lo - behind:hi - behind, h]
                    new = np.where(np.isfinite(new), np.clip(new, -MOST_VALUE[dtype], MOST_VALUE[dtype]), np.nan)
                    scale = scale_for(np.max(np.abs(new), initial=0, where=np.isfinite(new)), dtype)
                    if lo > at:
                        old = float(scales[page, h, block])
                        scale = max(scale, old)
                        if scale > old:
                            codes[page, h, slot:slot + lo - at] = nearest_code(CODE_VALUES[codes[page, h, slot:slot + lo - at]] * (old / scale))
                    codes[page, h, slot + lo - at:slot + hi - at] = nearest_code(new / scale)
                    scales[page, h, block] = scale
    return out


def values8(codes, scales, by_slot):
    """The values that pages in 8 bits stand for; by_slot: [page][head][slot][dim], otherwise [page][head][dim][slot]."""
    with np.errstate(invalid="ignore", over="ignore"):
        s = np.repeat(scales.astype(np.float64), 16, axis=2)
        return CODE_VALUES[codes] * (s[..., None] if by_slot else s[:, :, None])
