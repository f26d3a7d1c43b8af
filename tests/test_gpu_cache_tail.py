"""Attention of trees whose weights span more than half precision holds, in pieces of thousands of tokens.

The first token outweighs each other by e^gap, and the others' values are 2^16 times its own: the others make between 2^-12
(gap 28) and 2^-5.6 (24) of the result, though each weighs less than 2^-34.

What fp32 allows.  A weight is off by about 1e-6 (see test_gpu_cache), 5e-6 with room.  The weights' sum, to which the others
add less than 2^-21 in all, loses at most that, 5e-7.  An accumulator takes 16 tokens at a time, in up to three parts of
their weights, so 6 times a tile, and is off by less than a step of 2^-23 of itself each time, which way the matrix unit may
round: it does not round to the nearest, so such steps add up.  In all 5e-6 + 6 x 257 x 2^-23 = 1.9e-4.  Weights cut to 2^-37
of the largest would be off by a tenth of themselves at gap 24 and by all from 27 on: 2.2e-4 to 1.5e-3.

256 requests of two KV heads are as many as there are workers, so that a piece is a whole request.  They share their pages;
their queries differ.
"""
from __future__ import annotations

import numpy as np
import pytest
import torch

from oracle import bf16_bits_to_f64
from oracle import cache as oc
from oracle import tree as ot
from test_gpu_cache import FORMATS, IDS, Cache, _bits, _ints, _normal
from test_gpu_cache_tree import TreeRows
from tree_inputs import random_parents, words_of

pytestmark = pytest.mark.gpu

TOKENS = 8192


def _long(fmt, B, k, v):
    """A cache whose requests all read the same pages."""
    c = Cache(fmt, k.shape[1], 64, [len(k)])
    c.fill_tokens([len(k)], 5, k, v)
    c.table = np.repeat(c.table, B, 0)
    c.dtable = _ints(c.table)
    return c


def _errors(c, r, words, hq, some):
    """Relative 2-norm of the error of requests `some`, by KV head, and the largest error of their lse."""
    torch.cuda.synchronize()
    hkv, G = c.hkv, hq // c.hkv
    k, v, there = oc.tokens(c.pages, c.fmt, c.page, c.table, 0, max(r.end))
    assert there.all()
    out, lse, q = r.out.cpu().numpy().astype(np.float64), r.lse.cpu().numpy(), bf16_bits_to_f64(_bits(r.q))
    off, off_lse = [], 0.0
    for b in some:
        n, end = len(words[b]), r.end[b]
        seen = np.ones((n, end), bool)
        for i in range(n):
            seen[i, end - n:] = [words[b][i] >> j & 1 for j in range(n)]
        for h in range(hkv):
            mine = slice(r.start[b], r.start[b] + n), slice(h * G, (h + 1) * G)
            s = np.where(seen[:, None], np.einsum("ngd,td->ngt", q[mine], k[h, :end]) * r.scale, -np.inf)
            m = s.max(-1, keepdims=True)
            w = np.exp(s - m)
            l = w.sum(-1)
            with np.errstate(invalid="ignore"):
                want = (np.where(w > 0, w, 0) / l[..., None]) @ np.where(np.isfinite(v[h, :end]), v[h, :end], 0)
            off.append(np.linalg.norm(out[mine] - want) / np.linalg.norm(want))
            off_lse = max(off_lse, np.abs(lse[mine] - (m[..., 0] + np.log(l))).max())
    return off, off_lse


@pytest.mark.parametrize("fmt", FORMATS, ids=IDS.get)
@pytest.mark.parametrize("B,n", ((256, 16), (256, 24), (128, 64)), ids=("64rows", "96rows", "256rows"))
@pytest.mark.parametrize("gap", (24, 25, 26, 27, 28))
def test_small_weights_of_large_values(fmt, B, n, gap):
    hq, hkv = 8, 2
    rng = np.random.default_rng(gap)
    T = TOKENS + n
    k = 0.25 * _normal(5, T, hkv, 128)
    k[0] = 2.0
    v = 256 * (1 + 0.25 * _normal(6, T, hkv, 128).float()).to(torch.bfloat16)
    v[0] = 2.0 ** -8
    c = _long(fmt, B, k, v)
    q = (gap / (2 * 128 ** 0.5) * (1 + 0.25 * _normal(4, B * n, hq, 128).float())).to(torch.bfloat16)
    words = [words_of(random_parents(rng, n)) for _ in range(B)]
    r = TreeRows(c, hq, words, [T] * B, q=q).run()
    off, off_lse = _errors(c, r, words, hq, (0, 77, B - 1))
    assert max(off) <= 5e-6 + 6 * -(-T // 32) * 2.0 ** -23 and off_lse <= 5e-6 * max(1.0, gap)


@pytest.mark.parametrize("fmt", FORMATS, ids=IDS.get)
@pytest.mark.parametrize("window", (0, 5000))
@pytest.mark.parametrize("outlier", (0, 2.0 ** 12, 2.0 ** 100))
def test_weights_of_every_size_in_one_tile(fmt, window, outlier):
    """Large, small and tiny weights side by side in every tile, requests of one to 24 nodes, whole and in a window's parts; V
    blocks far beyond the others among them.

    Of 32 tokens one weighs e^-11 of the first (V 2^-4), 27 e^-26 (V 2^8, the first's 2^-8: 2e-3 of the result in all), four e^-45.
    A score is eight accumulations of 16 products of one sign, each off by a step at most: 8 x 2^-18 at 45, half of that at
    19; the exponent's scale and its rounding add 65 x 2^-23: weights are off by 6e-5 of each other.  The accumulators' steps come
    on top, as above.  Small weights lost would leave 2e-3 out.
    """
    hq, hkv, B = 8, 2, 256
    rng = np.random.default_rng(window)
    sizes = [(24, 1, 17, 5, 20, 16)[b % 6] for b in range(B)]
    T = TOKENS + 24
    # one level to a block of 32 channels, each exact in four bits; a score is 3.75 times their sum
    level = torch.tensor([1.5, 1.5, 1.0, 1.0]).repeat(T, 1)
    level[5::8] = 0.0
    level[::32] = torch.tensor([3.0, 2.0, 2.0, 2.0])
    level[0] = 3.0
    k = level.repeat_interleave(32, 1).to(torch.bfloat16).cuda()[:, None].expand(T, hkv, 128).contiguous()
    v = 256 * (1 + 0.25 * _normal(6, T, hkv, 128).float())
    v[::32] /= 4096
    v[0] = 2.0 ** -8
    if outlier:
        v[4000::2000, :, 32:64] *= outlier
    v = v.to(torch.bfloat16)
    c = _long(fmt, B, k, v)
    words = [words_of(random_parents(rng, n)) for n in sizes]
    q = (15 / 128 ** 0.5 * (1 + 0.0625 * _normal(4, sum(sizes), hq, 128).float())).to(torch.bfloat16)
    r = TreeRows(c, hq, words, [TOKENS + n for n in sizes], q=q, window=window, sinks=3 if window else 0).run()
    if window:
        torch.cuda.synchronize()
        end = [TOKENS + n for n in sizes]
        some = [0, 1, 2, 3, 255]
        out = r.out.cpu().numpy().astype(np.float64)
        kk, vv, _ = oc.tokens(c.pages, c.fmt, c.page, c.table, 0, T)
        qq = bf16_bits_to_f64(_bits(r.q))
        for b in some:
            for i in (0, sizes[b] - 1):
                row = r.start[b] + i
                live = np.array(ot.tree_sees(words[b][i], i, sizes[b], end[b], window, 3))
                for h in range(hkv):
                    s = qq[row, 4 * h:4 * h + 4] @ kk[h, live].T * r.scale
                    w = np.exp(s - s.max(-1, keepdims=True))
                    want = w / w.sum(-1, keepdims=True) @ vv[h, live]
                    for block in range(4):
                        g, x = out[row, 4 * h:4 * h + 4, 32 * block:32 * block + 32], want[:, 32 * block:32 * block + 32]
                        assert np.linalg.norm(g - x) <= (6e-5 + 6 * -(-T // 32) * 2.0 ** -23) * np.linalg.norm(x)
    else:
        off, off_lse = _errors(c, r, words, hq, (0, 1, 2, 3, 255))
        assert max(off) <= 6e-5 + 6 * -(-T // 32) * 2.0 ** -23 and off_lse <= 6e-5
