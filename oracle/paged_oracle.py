"""fp64 definitions of the paged-cache operators, for the tests: plain loops over sequences and tokens, numpy only."""
from __future__ import annotations

import numpy as np


def pair_axes(sections, order):
    """Axis of every rotary pair: section after section ("blocks"), or in turn by the axes that have pairs left ("turns")."""
    left, out = list(sections), []
    if order == "blocks":
        return [a for a, n in enumerate(left) for _ in range(n)]
    while any(left):
        for a in range(len(left)):
            if left[a]:
                out.append(a)
                left[a] -= 1
    return out


def rotate(x, positions, sections, base, layout, order="blocks", inverse=False):
    """x [n, heads, D], positions [axes, n]."""
    x = np.asarray(x, dtype=np.float64)
    d = x.shape[-1]
    axis = pair_axes(sections, order)
    out = np.empty_like(x)
    for i in range(d // 2):
        t = np.asarray(positions[axis[i]], dtype=np.float64) * float(base) ** (-2.0 * i / d) * (-1 if inverse else 1)
        a, b = (i, i + d // 2) if layout == "half" else (2 * i, 2 * i + 1)
        c, s = np.cos(t)[:, None], np.sin(t)[:, None]
        out[..., a] = x[..., a] * c - x[..., b] * s
        out[..., b] = x[..., a] * s + x[..., b] * c
    return out


def row_of(table_row, index, page_size):
    """(page, row) of an index of a sequence."""
    return table_row[index // page_size], index % page_size


def append(pages, rows, token_start, kv_len, table):
    """pages [n_pages, page_size, Hkv, D] with the new tokens' rows written."""
    pages = pages.copy()
    n_pages, size = pages.shape[:2]
    for s in range(len(kv_len)):
        n = token_start[s + 1] - token_start[s]
        for i in range(n):
            j = kv_len[s] - n + i
            if 0 <= j < len(table[s]) * size:
                page, row = row_of(table[s], j, size)
                if 0 <= page < n_pages:
                    pages[page, row] = rows[token_start[s] + i]
    return pages


def visible(p, n_keys, window, sinks):
    """Indexes that the token at index p sees."""
    return [j for j in range(min(p + 1, n_keys)) if window is None or p - j < window or j < sinks]


def attention(q, k_pages, v_pages, token_start, kv_len, table, scale, window=None, sinks=0, prefix_pages=(), n_prefix=0, every=1):
    """[n_tokens, Hq, D] and the same with |v| in the place of v (what a rounding of the probabilities can move); rows of
    no sequence are NaN, rows that see nothing 0.  every > 1: only so many tokens of a sequence, its first and last among them; the
    others are NaN too."""
    q = np.asarray(q, dtype=np.float64)
    size, hkv = k_pages.shape[1:3]
    g = q.shape[1] // hkv
    out, spread = np.full_like(q, np.nan), np.full_like(q, np.nan)
    first = [row_of(prefix_pages, j, size) for j in range(n_prefix)]
    for s in range(len(kv_len)):
        n = token_start[s + 1] - token_start[s]
        for i in sorted({*range(0, n, every), n - 1} if n else ()):
            p, t = kv_len[s] - n + i, token_start[s] + i
            at = first + [row_of(table[s], j, size) for j in visible(p, len(table[s]) * size, window, sinks)]
            out[t] = spread[t] = 0.0
            if not at:
                continue
            pages, rows = np.array(at).T
            k, v = k_pages[pages, rows].astype(np.float64), v_pages[pages, rows].astype(np.float64)     # [keys, Hkv, D]
            for h in range(q.shape[1]):
                w = k[:, h // g] @ q[t, h] * scale
                w = np.exp(w - w.max())
                w /= w.sum()
                out[t, h] = w @ v[:, h // g]
                spread[t, h] = w @ np.abs(v[:, h // g])
    return out, spread
