"""Drafted trees over the paged cache in numpy and float64: rows turned by their
positions, attention of a tree or in a window, and the accepted path kept.

bf16 values come as bit patterns (uint16).  Which tokens a row sees is listed
token by token from the definition; nothing here is shared with the HIP path.
"""
from __future__ import annotations

import numpy as np

from . import cache as oc
from .attention import bf16_bits_to_f64


def bf16_bits(x: np.ndarray) -> np.ndarray:
    """float64 -> the nearest bf16's bits, the even one of two (finite values within its range)."""
    m, e = np.frexp(x)
    e = np.maximum(e, -125)                                  # subnormal ones are multiples of 2^-133
    step = np.exp2((e - 8).astype(np.float64))
    y = (np.rint(x / step) * step).astype(np.float32)
    return (np.ascontiguousarray(y).view(np.uint32) >> 16).astype(np.uint16)


def turned(bits: np.ndarray, positions, inv_freq: np.ndarray, interleaved: bool = False, scale: float = 1.0) -> np.ndarray:
    """Rows [T, heads, 128] turned, in float64: pair j by position times inv_freq[j]."""
    x = bf16_bits_to_f64(bits).copy()
    f = inv_freq.astype(np.float64)
    half = len(f)
    for t, p in enumerate(positions):
        a = float(p) * f
        c, s = scale * np.cos(a), scale * np.sin(a)
        for j in range(half):
            i0, i1 = (2 * j, 2 * j + 1) if interleaved else (j, j + half)
            x0, x1 = x[t, :, i0].copy(), x[t, :, i1].copy()
            x[t, :, i0] = x0 * c[j] - x1 * s[j]
            x[t, :, i1] = x1 * c[j] + x0 * s[j]
    return x


def tree_sees(word: int, i: int, n: int, end: int, window: int = 0, sinks: int = 0):
    """Positions that row i of n sees: of the tokens before the tree those in the window or among the first, and
    the nodes whose bit is set."""
    first = end - n
    nodes = [j for j in range(n) if word >> j & 1]
    p = first + len(nodes) - 1
    past = [t for t in range(max(0, first)) if window == 0 or t > p - window or t < sinks]
    return past + [first + j for j in nodes if first + j >= 0]


def window_sees(i: int, n: int, end: int, window: int, sinks: int):
    """Positions that row i of n, a chain, sees."""
    p = end - n + i
    return [t for t in range(max(0, p + 1)) if t > p - window or t < sinks]


def attend(q_bits, pages, fmt, page, table, row_start, end, scale, sees, prev=None):
    """out [T, Hq, 128], lse [T, Hq] in float64; sees(row, i, n, end): positions; rows of no request are NaN."""
    T, hq, d = q_bits.shape
    hkv = pages.shape[1]
    out, lse = np.full((T, hq, d), np.nan), np.full((T, hq), np.nan)
    q = bf16_bits_to_f64(q_bits)
    for b in range(len(end)):
        n = int(row_start[b + 1] - row_start[b])
        if n <= 0:
            continue
        k, v, there = oc.tokens(pages, fmt, page, table, b, end[b])
        for i in range(n):
            row = int(row_start[b]) + i
            live = np.array([t for t in sees(row, i, n, int(end[b])) if 0 <= t < k.shape[1] and there[t]], np.int64)
            for h in range(hq):
                g = h // (hq // hkv)
                s = scale * (k[g, live] @ q[row, h])
                m = s.max() if len(s) else -np.inf
                if m == -np.inf and not np.isnan(s).any():
                    out[row, h], lse[row, h] = 0.0, -np.inf
                else:
                    with np.errstate(invalid="ignore"):
                        w = np.exp(s - m)
                        out[row, h], lse[row, h] = w @ v[g, live] / w.sum(), m + np.log(w.sum())
                if prev is not None:
                    po, pl = prev[0][row, h].astype(np.float64), float(prev[1][row, h])
                    if pl != -np.inf and lse[row, h] == -np.inf:
                        out[row, h], lse[row, h] = po, pl
                    elif pl != -np.inf:
                        both = np.logaddexp(lse[row, h], pl)
                        out[row, h] = out[row, h] * np.exp(lse[row, h] - both) + po * np.exp(pl - both)
                        lse[row, h] = both
    return out, lse


def keep(pages, fmt, page, table, kept, row_start, end):
    """pages after each request's kept nodes (a list of indices among its last tokens) moved to the front (a copy)."""
    before = oc.parts(pages, fmt, page)
    pages = pages.copy()
    after = oc.parts(pages, fmt, page)

    def place(b, pos):
        at = int(table[b][pos // page]) if 0 <= pos < table.shape[1] * page else -1
        return (at, pos % page) if 0 <= at < len(pages) else None

    for b, path in enumerate(kept):
        n = int(row_start[b + 1] - row_start[b])
        for j, node in enumerate(path[:n]):
            if not 0 <= node < n:
                continue
            old, new = place(b, int(end[b]) - n + node), place(b, int(end[b]) - n + j)
            if old is None or new is None:
                continue
            for src, dst in zip(before, after):
                dst[new[0], :, new[1]] = src[old[0], :, old[1]]
    return pages
