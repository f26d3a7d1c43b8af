"""Attention of 65 rows per KV head and more over 8- and 4-bit pages: V's scales and codes one by one, around the ends of half
precision.

V's values are bf16 numbers whatever their scale, so every value is exact and the tolerance is that of all attention
here, 5e-6 in the 2-norm (see test_gpu_cache), for each request and block of 32 channels by itself.  As f16 numbers, times 2^6
(e4m3) or 2^2 (e2m1), they would be exact from scale byte 106 to 128, or 102 to 138, at the lower end as subnormal numbers, which
the matrix unit adds with fewer bits: the smallest codes there were off by 5e-5.
"""
from __future__ import annotations

import numpy as np
import pytest
import torch

from oracle import cache as oc
from test_gpu_cache import IDS, Cache
from test_gpu_cache_tree import TreeRows, _trees

pytestmark = pytest.mark.gpu

ENDS = {oc.MXFP8: (106, 128), oc.MXFP4: (102, 138)}
SMALLEST = {oc.MXFP8: np.arange(1, 8), oc.MXFP4: np.array([1])}                     # subnormal ones
LARGEST = {oc.MXFP8: np.arange(0x70, 0x7F), oc.MXFP4: np.array([6, 7])}
ALL = {oc.MXFP8: np.arange(0x7F), oc.MXFP4: np.arange(8)}


def _set_v(c, b, tokens, codes, scales):
    """Codes [tokens, hkv, 128] and scale bytes [tokens, hkv, 4] of request b's first tokens."""
    V, VS = oc.parts(c.pages, c.fmt, c.page)[1::2]
    t = np.arange(tokens)
    at, slot = c.table[b][t // c.page], t % c.page
    V[at, :, slot] = codes if c.fmt == oc.MXFP8 else codes[..., 0::2] | codes[..., 1::2] << 4
    VS[at, :, slot] = scales


def _check(c, r, words):
    torch.cuda.synchronize()
    want, wl = r.want()
    got = r.out.cpu().numpy().astype(np.float64)
    for b in range(len(words)):
        mine = slice(r.start[b], r.start[b + 1])
        for h in range(c.hkv):
            heads = slice(h * r.hq // c.hkv, (h + 1) * r.hq // c.hkv)
            for block in range(4):
                g, x = got[mine, heads, 32 * block:32 * block + 32], want[mine, heads, 32 * block:32 * block + 32]
                assert np.linalg.norm(x) > 0 and np.linalg.norm(g - x) <= 5e-6 * np.linalg.norm(x), (b, h, block)
    assert np.abs(r.lse.cpu().numpy() - wl).max() <= 5e-6 * max(1.0, np.abs(wl).max())


@pytest.mark.parametrize("fmt", (oc.MXFP8, oc.MXFP4), ids=IDS.get)
@pytest.mark.parametrize("hq,n", ((8, 17), (8, 24), (16, 64)))
@pytest.mark.parametrize("which", (SMALLEST, LARGEST, ALL), ids=("smallest", "largest", "all"))
def test_scales_at_the_ends(fmt, hq, n, which):
    """A request for each scale: the two ends of the range, their neighbours inside and outside, and its middle."""
    rng = np.random.default_rng(n)
    low, high = ENDS[fmt]
    bytes_ = (low - 1, low, low + 1, 120, high - 1, high, high + 1)
    end = [70 + n] * len(bytes_)
    c = Cache(fmt, 2, 32, end)
    c.fill_tokens(end, 5)
    sign = {oc.MXFP8: 0x80, oc.MXFP4: 8}[fmt]
    for b, scale in enumerate(bytes_):
        codes = rng.choice(which[fmt], (end[b], 2, 128)) | sign * rng.integers(0, 2, (end[b], 2, 128))
        _set_v(c, b, end[b], codes.astype(np.uint8), np.full((end[b], 2, 4), scale, np.uint8))
    c.dev.copy_(torch.from_numpy(c.pages))
    words = _trees(rng, [n] * len(end))
    _check(c, TreeRows(c, hq, words, end).run(), words)


@pytest.mark.parametrize("fmt", (oc.MXFP8, oc.MXFP4), ids=IDS.get)
@pytest.mark.parametrize("hq,n", ((8, 24), (16, 64)))
def test_blocks_of_every_scale_in_one_tile(fmt, hq, n):
    """Channel blocks with scales of their own; tokens whose block lies beyond the range among those within, in the history and
    in the tree."""
    rng = np.random.default_rng(n)
    low, high = ENDS[fmt]
    end = [200 + n, 64 + n, n]
    c = Cache(fmt, 2, 32, end)
    c.fill_tokens(end, 5)
    block = np.array([low, high, 117, 124])
    for b, e in enumerate(end):
        scales = np.broadcast_to(block, (e, 2, 4)).copy()
        if b == 0:
            scales[40, 0, 0] = low - 3                       # below, one token
            scales[100:103, 1, 1] = high + 2                 # above
            scales[e - 2, 0, 2] = 127 + 30                   # far above, a node
        if b == 1:
            scales[::7, :, 3] = 16                           # the least that a write makes
        codes = rng.choice(ALL[fmt], (e, 2, 128)) | {oc.MXFP8: 0x80, oc.MXFP4: 8}[fmt] * rng.integers(0, 2, (e, 2, 128))
        _set_v(c, b, e, codes.astype(np.uint8), scales.astype(np.uint8))
    c.dev.copy_(torch.from_numpy(c.pages))
    words = _trees(rng, [n] * 3)
    _check(c, TreeRows(c, hq, words, end).run(), words)
