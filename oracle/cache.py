"""The paged cache in numpy and float64: what a page holds, and attention over it.

bf16 values come as bit patterns (uint16).  Nothing here is shared with the
HIP path or with the timed cases' plain form.
"""
from __future__ import annotations

import numpy as np

from .attention import bf16_bits_to_f64

BF16, MXFP8, MXFP4 = 0, 1, 2
ROW_BYTES = {BF16: 256, MXFP8: 128, MXFP4: 64}
SCALE_BYTES = {BF16: 0, MXFP8: 4, MXFP4: 4}
_BITS = {MXFP8: (4, 3, 7), MXFP4: (2, 1, 1)}      # exponent and fraction bits, bias
_TOP = {MXFP8: 448.0, MXFP4: 6.0}


def page_bytes(fmt: int, hkv: int, page: int) -> int:
    return hkv * page * 2 * (ROW_BYTES[fmt] + SCALE_BYTES[fmt])


def code_values(fmt: int) -> np.ndarray:
    """The number each code stands for (e4m3's 0x7F and 0xFF are NaN)."""
    eb, mb, bias = _BITS[fmt]
    out = []
    for c in range(1 << (1 + eb + mb)):
        e, f = (c >> mb) & ((1 << eb) - 1), (c & ((1 << mb) - 1)) / (1 << mb)
        x = f * 2.0 ** (1 - bias) if e == 0 else (1 + f) * 2.0 ** (e - bias)
        if fmt == MXFP8 and (c & 0x7F) == 0x7F:
            x = np.nan
        out.append(-x if c >> (eb + mb) else x)
    return np.array(out)


def encode(bits: np.ndarray, fmt: int):
    """Rows [..., 128] of bf16 bit patterns -> (bytes [..., row bytes], scale bytes [..., 4])."""
    if fmt == BF16:
        return np.ascontiguousarray(bits).view(np.uint8), np.zeros(bits.shape[:-1] + (0,), np.uint8)
    x = bf16_bits_to_f64(bits).reshape(bits.shape[:-1] + (4, 32))
    bad = ~np.isfinite(x).all(-1)
    x = np.where(bad[..., None], 0.0, x)
    peak = np.abs(x).max(-1)
    e = np.full(peak.shape, -111, np.int64)
    while True:                                  # the smallest exponent, by its definition
        small = peak > _TOP[fmt] * np.exp2(e.astype(np.float64))
        if not small.any():
            break
        e[small] += 1
    y = x * np.exp2(-e.astype(np.float64))[..., None]
    grid = code_values(fmt)
    grid = grid[: len(grid) // 2]
    grid = grid[~np.isnan(grid)]
    a = np.abs(y)
    hi = np.clip(np.searchsorted(grid, a), 0, len(grid) - 1)
    lo = np.maximum(hi - 1, 0)
    up, down = grid[hi] - a, a - grid[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    sign = (np.ascontiguousarray(bits).reshape(y.shape) >> 15).astype(np.int64)
    code = code + sign * (128 if fmt == MXFP8 else 8)
    code = np.where(bad[..., None], 0, code).astype(np.uint8).reshape(bits.shape)
    scales = np.where(bad, 255, e + 127).astype(np.uint8)
    if fmt == MXFP4:
        code = code[..., 0::2] | code[..., 1::2] << 4
    return code, scales


def decode(rows: np.ndarray, scales: np.ndarray, fmt: int) -> np.ndarray:
    """What rows of a page stand for, in float64 [..., 128]."""
    if fmt == BF16:
        return bf16_bits_to_f64(np.ascontiguousarray(rows).view(np.uint16))
    if fmt == MXFP4:
        rows = np.stack([rows & 15, rows >> 4], -1).reshape(rows.shape[:-1] + (128,))
    f = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127))
    return code_values(fmt)[rows] * np.repeat(f, 32, -1)


def parts(pages: np.ndarray, fmt: int, page: int):
    """Views of pages [n, Hkv, block bytes]: K rows, V rows, K scales, V scales, each [n, Hkv, page, bytes]."""
    rb, sb = ROW_BYTES[fmt], SCALE_BYTES[fmt]
    cut = np.cumsum([0, page * rb, page * rb, page * sb, page * sb])
    return [pages[:, :, cut[i]:cut[i + 1]].reshape(pages.shape[0], pages.shape[1], page, -1) for i in range(4)]


def row_places(row_start, end, table, page, num_pages):
    """Of every row: (request, page, slot), page -1 where its token has no place; None for a row of no request."""
    places = [None] * int(row_start[-1])
    for b in range(len(end)):
        n = row_start[b + 1] - row_start[b]
        for i in range(n):
            pos = int(end[b]) - n + i
            at = int(table[b][pos // page]) if 0 <= pos < table.shape[1] * page else -1
            places[row_start[b] + i] = (b, at if 0 <= at < num_pages else -1, pos % page)
    return places


def write(pages, fmt, page, table, k_bits, v_bits, row_start, end):
    """pages after rows [T, Hkv, 128] were written (a copy)."""
    pages = pages.copy()
    K, V, KS, VS = parts(pages, fmt, page)
    assert K.base is not None and np.shares_memory(K, pages)
    kc, ks = encode(k_bits, fmt)
    vc, vs = encode(v_bits, fmt)
    for t, place in enumerate(row_places(row_start, end, table, page, len(pages))):
        if place is not None and place[1] >= 0:
            _, at, slot = place
            K[at, :, slot], V[at, :, slot], KS[at, :, slot], VS[at, :, slot] = kc[t], vc[t], ks[t], vs[t]
    return pages


def tokens(pages, fmt, page, table, b, upto):
    """K and V of request b's tokens [0, upto) as float64 [Hkv, upto, 128], and which of them exist."""
    K, V, KS, VS = parts(pages, fmt, page)
    upto = max(0, min(int(upto), table.shape[1] * page))
    pos = np.arange(upto)
    at = table[b][pos // page]
    there = (at >= 0) & (at < len(pages))
    at = np.where(there, at, 0)
    k = decode(K[at, :, pos % page], KS[at, :, pos % page], fmt)
    v = decode(V[at, :, pos % page], VS[at, :, pos % page], fmt)
    return k.transpose(1, 0, 2), v.transpose(1, 0, 2), there


def attend(q_bits, pages, fmt, page, table, row_start, end, scale, causal, prev=None):
    """out [T, Hq, 128], lse [T, Hq] in float64; rows of no request are NaN."""
    T, hq, d = q_bits.shape
    hkv = pages.shape[1]
    out, lse = np.full((T, hq, d), np.nan), np.full((T, hq), np.nan)
    q = bf16_bits_to_f64(q_bits)
    for b in range(len(end)):
        n = row_start[b + 1] - row_start[b]
        if n <= 0:
            continue
        k, v, there = tokens(pages, fmt, page, table, b, end[b])
        for i in range(n):
            sees = min(k.shape[1], max(0, int(end[b]) - n + i + 1)) if causal else k.shape[1]
            live = np.nonzero(there[:sees])[0]
            row = row_start[b] + i
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
