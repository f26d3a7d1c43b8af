"""The paged cache's attention with 17 to 64 rows per KV head (the 32-row products) where it can go wrong: lengths around
tiles and pages, pages that are none, leftovers in pages, joins; workgroups, pairs of waves, and waves by themselves.

Errors: the text of ``test_gpu_cache``; with an earlier part those of its weights too, 8e-6 of the largest value, 5."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from oracle import cache as oc
from test_gpu_cache import FORMATS, IDS, Cache, Rows, _ints

pytestmark = pytest.mark.gpu

WIDE = ((16, 3), (16, 8))        # query heads over 2 KV heads, rows: 24 and 64 per KV head


@pytest.mark.parametrize("fmt", FORMATS, ids=IDS.get)
@pytest.mark.parametrize("page", (16, 32, 64, 128, 256))
@pytest.mark.parametrize("hq,n", WIDE)
@pytest.mark.parametrize("causal", (0, 1))
def test_lengths(fmt, page, hq, n, causal):
    end = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 700, 3]
    rows = [1 + (5 * b + n) % n for b in range(len(end))]
    rows[6], rows[17], rows[18] = n, n, n
    c = Cache(fmt, 2, page, end)
    c.fill_tokens(end, 9)
    Rows(c, hq, rows, end, causal=causal, max_rows=n).run().check()


@pytest.mark.parametrize("fmt", FORMATS, ids=IDS.get)
@pytest.mark.parametrize("page", (16, 64))
@pytest.mark.parametrize("hq,n", WIDE)
def test_pages_that_are_none(fmt, page, hq, n):
    """Holes of a page number below or above the cache's: with pages of 16 one half of a tile, either one."""
    held = [200, 256, 100, 256, 0, 250]
    c = Cache(fmt, 2, page, held)
    c.fill_tokens(held, 5)
    c.table[0, 1], c.table[1, 0], c.table[2, :] = -1, c.num_pages, -7
    c.table[3, :-1] = 1 << 30
    c.table[5, 1::4], c.table[5, 2::4] = -1, c.num_pages + 1
    c.dtable = _ints(c.table)
    end = [200, 300, 100, 5000, -4, 250]
    for causal in (0, 1):
        Rows(c, hq, [n, max(1, n - 1), 1, n, 2, n], end, causal=causal).run().check()


@pytest.mark.parametrize("fmt", FORMATS, ids=IDS.get)
@pytest.mark.parametrize("fill", (0xFF, 0x7F, 0x80))
@pytest.mark.parametrize("hq,n", WIDE)
def test_leftovers_in_pages(fmt, fill, hq, n):
    end = [1, 17, 45, 97]
    c = Cache(fmt, 2, 64, end, fill=fill)
    c.fill_tokens(end, 5)
    Rows(c, hq, [1, 2, n, n - 1], end).run().check()


@pytest.mark.parametrize("fmt", FORMATS, ids=IDS.get)
@pytest.mark.parametrize("hq,n", WIDE)
def test_joined(fmt, hq, n):
    end, rows = [300, 0, 64, 0], [n, 2, 1, n]
    c = Cache(fmt, 2, 32, end)
    c.fill_tokens(end, 5)
    T = sum(rows)
    po, pl = torch.randn(T, hq, 128, generator=torch.Generator().manual_seed(1)).cuda(), (torch.rand(T, hq, generator=torch.Generator().manual_seed(2)) * 12 - 2).cuda()
    for t in (1, n, T - 1):                          # nothing came before: of a row with tokens, and of two without
        pl[t], po[t] = float("-inf"), float("nan")
    r = Rows(c, hq, rows, end, prev=(po, pl)).run()
    r.check(r._bound() + 8e-6 * 5)


@pytest.mark.parametrize("fmt", FORMATS, ids=IDS.get)
@pytest.mark.parametrize("hkv,hq,n", ((8, 16, 3), (8, 64, 3)))
def test_waves_alone(fmt, hkv, hq, n):
    """1040 (request, head) pairs, 6 and 24 rows per KV head: holes in either half of a tile, leftovers, a long request."""
    rng = np.random.default_rng(7)
    end = rng.integers(0, 80, 130)
    end[64], end[129] = 900, 33
    c = Cache(fmt, hkv, 16, end, fill=0xFF)
    c.fill_tokens(end, 3)
    drop = rng.random(c.table.shape) < 0.2
    drop[64] = False
    drop[64, 5::7] = True
    c.table[drop] = -1
    c.dtable = _ints(c.table)
    Rows(c, hq, rng.integers(0, n + 1, 130), end, max_rows=n).run().check()
